// Verification of drafted tokens against the target's distribution, on the sampler's integer weights (sampler.cuh).
//
// A sequence's drafts form a tree; node 0 is the token that is already accepted.  At a node with kept weights a_i (the
// sampler's w_i inside its nucleus, 0 outside) of mass A = sum a_i the children are tested in order of their rows:
//   d_i = floor(q_i A)     with the draft's probabilities q (one product in 64 bits), or A at the child's token and 0 elsewhere
//   accepted when (d_x u24) >> 24 < a_x,  x the child's token; the walk goes on there
//   refused: a_i becomes max(a_i - d_i, 0) (unless nothing would be left: then a stays), the next child is tested
// and where no child is left the next token is the first whose running sum of a exceeds (A u24) >> 24.  All integers but the
// product, so that decisions do not depend on the order of sums; each emitted token is distributed as the sampler's.
//
// Only the nodes on the accepted path are looked at, one after the other.  A cluster of C CTAs holds a node's row as weights
// in its shared memory (one read of the logits), so that maximum, sums, nucleus, tests, differences and the inverse
// CDF are passes over shared memory with one cluster barrier each.  The nucleus is found with exact mass histograms: first 256
// buckets of the exponent and three more bits, so that the elements spread over them whatever the temperature, then nine
// bits at a time.
#pragma once
#include "attn_tc.cuh"
#include "cache_evict.cuh"
#include "sampler.cuh"

namespace rpo {

struct VerifyArgs {
  const float* logits; int64_t logits_stride;
  const float* probs; int64_t probs_stride;       // NULL: drafts without probabilities
  const int32_t *tokens, *parents, *offsets;
  const float* uniform;
  int32_t *path, *n_path, *next;
  float* logprobs;                                // NULL, or like path
  int V, n_rows, max_path, greedy, eos_id, slice; // slice: words of a row per CTA
  float temperature; uint32_t top_p24;
  int* status;
};

constexpr int VF_THREADS = 512, VF_WARPS = VF_THREADS / 32;
constexpr int VF_B1 = 256, VF_COPIES = 8, VF_B2 = 512, VF_BITS = 9;
constexpr int VF_HIST = VF_B1 * VF_COPIES * 8 + 2 * VF_B2 * 8;

struct MassPair { uint32_t lo, hi; };             // sums of the lower 16 bits and of the others

__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t addr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}

// Bucket of a weight >= 1: exponent and three bits below it (monotone).
__device__ __forceinline__ int verify_bucket(uint32_t w) {
  const int e = 31 - __clz(w);
  return e * 8 + (e >= 3 ? (w >> (e - 3)) & 7 : (w << (3 - e)) & 7);
}

__device__ __forceinline__ uint32_t verify_u24(float u) {
  return u > 0.f ? min(__float2uint_rz(u * 16777216.f), (1u << 24) - 1) : 0u;
}

// floor(q A), 0 for what is no probability.
__device__ __forceinline__ uint64_t verify_scaled(float q, double mass) {
  return q > 0.f ? (uint64_t)__double2ull_rz(fmin(__dmul_rn((double)q, mass), 4.0e18)) : 0ull;
}

template <int C>
__global__ void __launch_bounds__(VF_THREADS) verify_kernel(VerifyArgs a) {
  extern __shared__ __align__(16) uint8_t vf_smem[];
  uint64_t* h1 = reinterpret_cast<uint64_t*>(vf_smem);                   // [bucket][copy] as MassPair, then copy 0 as the bucket's mass
  uint64_t* h2 = h1 + VF_B1 * VF_COPIES;                                  // two buffers of VF_B2
  uint32_t* wt = reinterpret_cast<uint32_t*>(vf_smem + (a.top_p24 < (1u << 24) ? VF_HIST : 0));     // this CTA's weights
  __shared__ uint64_t s_slot[2][2], s_red[VF_WARPS], s_bcast[4], s_wsum[VF_WARPS];
  __shared__ float s_sume[VF_WARPS];
  __shared__ int s_bin, s_child, s_token;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % C, s = blockIdx.x / C, V = a.V;
  const int c0 = min(V, rank * a.slice), n = min(V, c0 + a.slice) - c0;   // my words [c0, c0 + n)
  const int chunk = ((a.slice + VF_WARPS - 1) / VF_WARPS + 3) & ~3;       // of a warp
  const int w0 = min(n, warp * chunk), w1 = min(n, w0 + chunk);
  int32_t* path = a.path + (int64_t)s * a.max_path;
  float* logp = a.logprobs ? a.logprobs + (int64_t)s * a.max_path : nullptr;

  int row0 = a.offsets[s], rows = a.offsets[s + 1];
  if (row0 < 0 || rows < row0 || rows > a.n_rows) { if (tid == 0) atomicOr(a.status, STATUS_BAD_LENGTH); }
  row0 = min(max(row0, 0), a.n_rows);
  rows = min(max(rows - row0, 0), a.n_rows - row0);

  int turn = 0;                                   // exchanges so far: s_slot is used in turns
  auto remote = [&](const void* p, int r) { return fa::map_rank((uint32_t)__cvta_generic_to_shared(p), r); };
  // Sum (or maximum) over the CTAs of one or two words that thread 0 of each holds.
  auto exchange = [&](uint64_t x, uint64_t y, bool is_max, uint64_t* y_out) {
    const int b = turn++ & 1;
    if (tid == 0) { s_slot[b][0] = x; s_slot[b][1] = y; }
    fa::cluster_sync();
    if (warp == 0) {
      uint64_t u = lane < C ? ld_cluster_u64(remote(&s_slot[b][0], lane)) : 0, v = lane < C ? ld_cluster_u64(remote(&s_slot[b][1], lane)) : 0;
#pragma unroll
      for (int o = C / 2; o > 0; o >>= 1) {
        const uint64_t u2 = __shfl_xor_sync(0xffffffffu, u, o);
        u = is_max ? (u2 > u ? u2 : u) : u + u2;
        v += __shfl_xor_sync(0xffffffffu, v, o);
      }
      if (lane == 0) { s_bcast[0] = u; s_bcast[1] = v; }
    }
    __syncthreads();
    const uint64_t r = s_bcast[0];
    if (y_out) *y_out = s_bcast[1];
    __syncthreads();
    return r;
  };
  auto block_max = [&](uint64_t v) {              // valid in thread 0
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { const uint64_t x = __shfl_xor_sync(0xffffffffu, v, o); v = x > v ? x : v; }
    if (lane == 0) s_red[warp] = v;
    __syncthreads();
    if (warp == 0) {
      v = lane < VF_WARPS ? s_red[lane] : 0;
#pragma unroll
      for (int o = VF_WARPS / 2; o > 0; o >>= 1) { const uint64_t x = __shfl_xor_sync(0xffffffffu, v, o); v = x > v ? x : v; }
    }
    return v;
  };
  // Warps leave their sums in s_wsum; their sum, valid in thread 0.
  auto block_sum = [&](uint64_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (lane == 0) s_wsum[warp] = v;
    __syncthreads();
    uint64_t t = 0;
    if (tid == 0)
      for (int w = 0; w < VF_WARPS; ++w) t += s_wsum[w];
    return t;
  };
  // Among nb buckets with `mass(b)` over all CTAs: the highest with above + (mass of the buckets from it on) >= target.
  // (nb <= VF_THREADS; every CTA finds the same.)  *above grows by the mass above it.
  auto select = [&](const uint64_t* hist, int stride, int nb, uint64_t target, uint64_t* above, uint64_t* at) {
    const int b = nb - 1 - tid;
    uint64_t m = 0;
    if (b >= 0) {
#pragma unroll
      for (int r = 0; r < C; ++r) m += ld_cluster_u64(remote(hist + b * stride, r));
    }
    const uint64_t incl = warp_incl_scan_u64(m, lane);
    if (tid == 0) s_bin = -1;
    if (lane == 31) s_red[warp] = incl;
    __syncthreads();
    uint64_t run = *above + incl - m;
    for (int w = 0; w < warp; ++w) run += s_red[w];
    if (b >= 0 && m > 0 && run + m >= target) atomicMax(&s_bin, b);
    __syncthreads();
    const int bin = s_bin;
    if (b == bin) { s_bcast[2] = run; s_bcast[3] = m; }
    __syncthreads();
    *above = s_bcast[2]; *at = s_bcast[3];
    __syncthreads();
    return bin;
  };

  const bool vec = ((a.logits_stride & 3) == 0) && (((uintptr_t)a.logits & 15) == 0);
  const bool unit_T = a.temperature == 1.0f;
  int cur = 0, count = 0, next = -1;
  bool live = rows > 0;
  for (; live && count < a.max_path; ) {
    const int node_row = row0 + cur, token_here = a.tokens[node_row];
    if (rank == 0 && tid == 0) path[count] = cur;
    if (a.eos_id >= 0 && token_here == a.eos_id) {
      if (rank == 0 && tid == 0 && logp) logp[count] = 0.f;
      ++count;
      break;
    }
    // ---- the row's logits into shared memory, their maximum (lowest token among equal ones)
    const float* row = a.logits + (int64_t)node_row * a.logits_stride;
    float best = -INFINITY; int best_c = 0x7FFFFFFF;
    auto see = [&](int i, float x) {
      x = x < INFINITY ? x : -INFINITY;           // what is no number, or too large, counts as excluded
      if (x > best) { best = x; best_c = c0 + i; }
      return __float_as_uint(x);
    };
    if (vec) {
      for (int i = w0 + lane * 4; i < w1; i += 128) {
        if (i + 3 < w1) {
          const float4 x = *reinterpret_cast<const float4*>(row + c0 + i);
          uint4 y;
          y.x = see(i, x.x); y.y = see(i + 1, x.y); y.z = see(i + 2, x.z); y.w = see(i + 3, x.w);
          *reinterpret_cast<uint4*>(wt + i) = y;
        } else {
          for (int j = i; j < w1; ++j) wt[j] = see(j, row[c0 + j]);
        }
      }
    } else {
      for (int i = w0 + lane; i < w1; i += 32) wt[i] = see(i, row[c0 + i]);
    }
    uint64_t key = 0;
    if (best_c != 0x7FFFFFFF) {
      const uint32_t b = __float_as_uint(best + 0.0f);
      key = ((uint64_t)((b & 0x80000000u) ? ~b : (b | 0x80000000u)) << 32) | (0xFFFFFFFFu - (uint32_t)best_c);
    }
    key = exchange(block_max(key), 0, true, nullptr);
    const int argmax = key ? (int)(0xFFFFFFFFu - (uint32_t)key) : -1;
    const uint32_t ord = (uint32_t)(key >> 32);
    const float top = key ? __uint_as_float((ord & 0x80000000u) ? (ord & 0x7FFFFFFFu) : ~ord) : 0.f;
    const float zmax = unit_T ? top : __fdiv_rn(top, a.temperature);
    const bool nucleus = a.top_p24 < (1u << 24) && !a.greedy;
    // ---- weights, their sum, and the sum of the exponentials for the log-probability
    if (nucleus) {
      for (int i = tid; i < VF_B1 * VF_COPIES; i += VF_THREADS) h1[i] = 0;
      __syncthreads();
    }
    uint64_t tot = 0;
    float sume = 0.f;
    for (int i = w0 + lane; i < w1; i += 32) {
      const float x = __uint_as_float(wt[i]);
      const float e = key ? exp_nonpos(radd(unit_T ? x : __fdiv_rn(x, a.temperature), -zmax)) : 0.f;
      sume += e;
      const uint32_t w = a.greedy ? (c0 + i == argmax ? 1u : 0u) : __float2uint_rz(rmul(e, 1073741824.0f));
      wt[i] = w;
      tot += w;
      if (nucleus && w) {
        MassPair* h = reinterpret_cast<MassPair*>(h1) + verify_bucket(w) * VF_COPIES + (lane & (VF_COPIES - 1));
        atomicAdd(&h->lo, w & 0xFFFFu);
        if (w >> 16) atomicAdd(&h->hi, w >> 16);
      }
    }
    sume = warp_sum(sume);
    if (lane == 0) s_sume[warp] = sume;
    const uint64_t mine = block_sum(tot);
    float sum_cta = 0.f;
    if (tid == 0)
      for (int w = 0; w < VF_WARPS; ++w) sum_cta += s_sume[w];
    if (nucleus) {                                // (block_sum's barriers: the histogram is complete)
      if (tid < VF_B1) {
        uint64_t m = 0;
#pragma unroll
        for (int k = 0; k < VF_COPIES; ++k) { const MassPair p = reinterpret_cast<MassPair*>(h1)[tid * VF_COPIES + k]; m += p.lo + ((uint64_t)p.hi << 16); }
        h1[tid * VF_COPIES] = m;
      }
    }
    uint64_t sum_fixed;                           // of the exponentials, in units of 2^-40 (each CTA's float sum rounded once)
    uint64_t mass = exchange(mine, (uint64_t)__float2ull_rn(sum_cta * 1099511627776.f), false, &sum_fixed);
    uint32_t tau = 1;
    if (nucleus && mass) {
      const uint64_t target = mul_shift24(mass, a.top_p24);
      uint64_t above = 0, at = 0;
      const int b1 = select(h1, VF_COPIES, VF_B1, target, &above, &at);
      // b1: exponent e and three bits; the bits below in steps of nine
      const int e = b1 >> 3;
      int rest = max(e - 3, 0);
      uint32_t pre = e >= 3 ? 8u | (b1 & 7) : (8u | (b1 & 7)) >> (3 - e);       // the weight's leading bits so far
      for (int round = 0; rest > 0; ++round) {
        const int bits = min(rest, VF_BITS);
        uint64_t* h = h2 + (round & 1) * VF_B2;
        for (int i = tid; i < VF_B2; i += VF_THREADS) h[i] = 0;
        __syncthreads();
        for (int i = w0 + lane; i < w1; i += 32) {
          const uint32_t w = wt[i];
          if (w >> rest == pre) {
            MassPair* p = reinterpret_cast<MassPair*>(h) + ((w >> (rest - bits)) & ((1u << bits) - 1));
            atomicAdd(&p->lo, w & 0xFFFFu);
            if (w >> 16) atomicAdd(&p->hi, w >> 16);
          }
        }
        __syncthreads();
        for (int i = tid; i < VF_B2; i += VF_THREADS) { const MassPair p = reinterpret_cast<MassPair*>(h)[i]; h[i] = p.lo + ((uint64_t)p.hi << 16); }
        fa::cluster_sync();
        const int bin = select(h, 1, 1 << bits, target, &above, &at);
        pre = (pre << bits) | bin;
        rest -= bits;
      }
      tau = pre;
      mass = above + at;
    }
    // ---- children
    int accepted = -1, token = -1;
    bool lazy = false, sums = !nucleus;           // lazy: a - d with the last test's mass is what is left; sums: s_wsum holds it by warps
    double lazy_mass = 0;
    auto value = [&](int i) -> uint32_t {         // what is left of word i
      const uint32_t w = wt[i];
      return w >= tau ? w : 0u;
    };
    const float* q = a.probs ? a.probs + (int64_t)node_row * a.probs_stride : nullptr;
    auto less = [&](int i, double m) -> uint32_t {
      const uint32_t w = value(i);
      if (!w) return 0u;
      const uint64_t d = verify_scaled(q[c0 + i], m);
      return d < w ? w - (uint32_t)d : 0u;
    };
    bool refused = false;                         // drafts without probabilities: some child was refused
    for (int last = cur; count + 1 < a.max_path; ) {
      // the next child: all CTAs' first warps look for it
      if (warp == 0) {
        int child = -1;
        for (int j = last + 1; j < rows; j += 32) {
          const unsigned hit = __ballot_sync(0xffffffffu, j + lane < rows && a.parents[row0 + j + lane] == cur);
          if (hit) { child = j + __ffs(hit) - 1; break; }
        }
        if (lane == 0) s_child = child;
      }
      __syncthreads();
      const int child = s_child;
      if (child < 0) break;
      last = child;
      if (lazy) {                                 // make what the last test left the weights
        for (int i = w0 + lane; i < w1; i += 32) wt[i] = less(i, lazy_mass);      // (nobody reads them for that test any more)
        tau = 1; lazy = false;
        fa::cluster_sync();
      }
      if (warp == 0) {
        const int x = a.tokens[row0 + child];
        const bool in = x >= 0 && x < V;
        if (!in && lane == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
        uint64_t w = 0;
        if (in) {
          uint32_t y;
          asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(y) : "r"(remote(wt + x % a.slice, x / a.slice)) : "memory");
          w = y >= tau ? y : 0;
        }
        uint64_t d = mass;
        if (q) d = in ? verify_scaled(q[x], (double)mass) : 0;
        else {                                    // a token that was refused before has nothing left
          bool again = false;
          for (int j = cur + 1; j < child; j += 32)
            again = again || __any_sync(0xffffffffu, j + lane < child && a.parents[row0 + j + lane] == cur && a.tokens[row0 + j + lane] == x);
          if (again) w = 0;
        }
        const bool yes = mul_shift24(d, verify_u24(a.uniform[row0 + child])) < w;
        if (lane == 0) { s_bcast[2] = w; s_bcast[3] = yes; s_token = x; }
      }
      __syncthreads();
      const uint64_t w = s_bcast[2];
      if (s_bcast[3]) { accepted = child; token = s_token; }
      __syncthreads();
      if (accepted >= 0) break;
      if (!q) {
        if (w < mass) mass -= w;                  // (all of it is never refused)
        refused = true;
      } else {
        uint64_t left = 0;
        const double m = (double)mass;
        for (int i = w0 + lane; i < w1; i += 32) left += less(i, m);
        left = exchange(block_sum(left), 0, false, nullptr);
        if (left) { mass = left; lazy = true; lazy_mass = m; sums = true; }
        else sums = false;
      }
    }
    // ---- without an accepted child: the next token
    if (accepted < 0 && mass) {
      if (refused) {
        fa::cluster_sync();                       // nobody reads the refused tokens' weights any more
        for (int j = cur + 1 + tid; j < rows; j += VF_THREADS)
          if (a.parents[row0 + j] == cur) { const int x = a.tokens[row0 + j] - c0; if (x >= 0 && x < n) wt[x] = 0; }
        __syncthreads();
        sums = false;
      }
      uint64_t local = 0;
      auto left = [&](int i) { return lazy ? less(i, lazy_mass) : value(i); };
      if (!sums) {
        for (int i = w0 + lane; i < w1; i += 32) local += left(i);
        local = block_sum(local);
      } else if (tid == 0) {
        for (int w = 0; w < VF_WARPS; ++w) local += s_wsum[w];
      }
      // mass in the CTAs before mine
      const int b = turn++ & 1;
      if (tid == 0) { s_slot[b][0] = local; s_token = -1; }
      fa::cluster_sync();
      uint64_t base = 0, r = mul_shift24(mass, verify_u24(a.uniform[row0]));
      for (int k = 0; k < rank; ++k) base += ld_cluster_u64(remote(&s_slot[b][0], k));
      for (int w = 0; w < warp; ++w) base += s_wsum[w];
      if (r >= base && r < base + s_wsum[warp]) {          // one warp of the cluster
        for (int i = w0; i < w1; i += 128) {
          uint32_t x[4];
          uint64_t sum = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) { x[k] = i + lane * 4 + k < w1 ? left(i + lane * 4 + k) : 0u; sum += x[k]; }
          const uint64_t incl = warp_incl_scan_u64(sum, lane);
          const unsigned hit = __ballot_sync(0xffffffffu, base + incl > r);
          if (hit) {
            if (lane == __ffs(hit) - 1) {
              uint64_t run = base + incl - sum;
              int k = 0;
              while (k < 3 && run + x[k] <= r) run += x[k++];
              const int tok = c0 + i + lane * 4 + k;
              a.next[s] = tok;
              if (logp) logp[count] = radd(unit_T ? row[tok] : __fdiv_rn(row[tok], a.temperature), -zmax) - logf((float)sum_fixed * (1.f / 1099511627776.f));
            }
            break;
          }
          base += __shfl_sync(0xffffffffu, incl, 31);
        }
      }
      next = 0;                                   // written above
    } else if (rank == 0 && tid == 0) {
      if (logp) logp[count] = accepted < 0 ? -INFINITY
          : radd(unit_T ? row[token] : __fdiv_rn(row[token], a.temperature), -zmax) - logf((float)sum_fixed * (1.f / 1099511627776.f));
    }
    ++count;
    live = accepted >= 0;
    cur = accepted;
    if (live) fa::cluster_sync();                 // nobody reads this row's weights any more
  }
  if (rank == 0) {
    if (tid == 0) { a.n_path[s] = count; if (next < 0) a.next[s] = -1; }
    for (int i = count + tid; i < a.max_path; i += VF_THREADS) { path[i] = -1; if (logp) logp[i] = 0.f; }
  }
  fa::cluster_sync();                             // no CTA leaves while another reads its shared memory
}

}  // namespace rpo
