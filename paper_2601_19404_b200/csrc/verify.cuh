// Verification of drafted tokens against the target's distribution, on the sampler's integer weights (sampler.cuh).
//
// A sequence's drafts form a tree; node 0 is the token that is already accepted.  At a node with kept weights a_i (the
// sampler's w_i inside its nucleus, 0 outside) of mass A = sum a_i the children are tested in order of their rows:
//   d_i = floor(q_i A)     with the draft's probabilities q (one product in 64 bits), or A at the child's token and 0 elsewhere
//   accepted when (d_x u24) >> 24 < a_x,  x the child's token; the walk goes on there
//   refused: a_i becomes max(a_i - d_i, 0) (unless nothing would be left: then a stays), the next child is tested
// A child with a negative token is passed over; one beyond the vocabulary has a_x = 0, so it is refused as any other.
// Where no child is left the next token is the first whose running sum of a exceeds (A u24) >> 24.  All integers but the
// product, so that decisions do not depend on the order of sums; each emitted token is distributed as the sampler's.
//
// Only the nodes on the accepted path are looked at, one after the other.  A cluster of C CTAs holds a node's row as weights
// in its shared memory (one read of the logits), so that maximum, sums, nucleus, tests, differences and the inverse
// CDF are passes over shared memory with one cluster barrier each.  The nucleus is found with exact mass histograms: first 256
// buckets of the exponent and three more bits, so that the elements spread over them whatever the temperature, then nine
// bits at a time.  It is found only where something depends on it: a draft that the whole row's mass would accept, and whose
// weight has less than the nucleus's share above it, is accepted without (one sum instead of the search).
//
// Bound by instructions and barriers, not by HBM: a row of 152064 costs a cluster 13 000 clocks without the nucleus (2900 fetch, 3700
// exponentials, two exchanges of 2000, the test 1000), the nucleus 15 000, the difference with q 4000 to 6000.  128 chains of 9 with
// probabilities, nucleus 0.95, 2.96 rows looked at on average, nine at most: 240 to 262 us (floor 41 us for their bytes).  Steps: scalar loads
// and weights 764; loads in flight, sums pushed through the cluster 662; two CTAs per SM 398; columns for the histograms 369; accepted
// drafts without the nucleus 275; packed arithmetic 247.  256 threads rather than 512: every warp repeats the decisions.
// 4 trees of 24 without probabilities, five levels at most: 22 to 37 us.
#pragma once
#include <type_traits>

#include "attn_tc.cuh"
#include "paged_chunk.cuh"
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

constexpr int VF_THREADS = 256, VF_WARPS = VF_THREADS / 32;
constexpr int VF_B1 = 256, VF_COPIES = 4, VF_B2 = 512, VF_BITS = 9, VF_COLUMN = 12, VF_KEPT = VF_COLUMN * 32;
// With the weights of 2^17 tokens and more two CTAs still fit an SM.
constexpr int VF_HIST = VF_B1 * VF_COPIES * 8 + VF_B1 * 8 + 2 * VF_B2 * 8 + VF_WARPS * VF_KEPT * 4;
constexpr int VF_NODES = 128;                     // what concerns so many nodes is gathered in shared memory at the start

struct MassPair { uint32_t lo, hi; };             // sums of the lower 16 bits and of the others
struct VerifyNode { int parent, token; uint32_t u24; float q, logit; };       // q, logit: of its token, in its parent's rows

__device__ __forceinline__ uint32_t verify_u24(float u) {
  return u > 0.f ? min(__float2uint_rz(u * 16777216.f), (1u << 24) - 1) : 0u;
}

// q A of a probability, 0 for what is none; its whole part is what a test takes (2^62 at most: more than any weight, whatever it
// is multiplied by).
__device__ __forceinline__ double verify_scaled(float q, double mass) { return __dmul_rn((double)(q > 0.f ? fminf(q, 16384.f) : 0.f), mass); }

// exp_nonpos(x) 2^30 of two numbers, with the same roundings in fewer instructions: packed additions and products, rint by adding
// 1.5 x 2^23 (and 30), whose low bits then are the exponent that the polynomial's result is raised by.  Numbers below -40 count as -40:
// between there and -24 the sampler's exponential is 0, this one below 2^-4, which is a weight of 0 too and nothing in a sum.
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ void verify_exp(float x0, float x1, float& e0, float& e1) {
  constexpr float shift = 12582912.0f + 30.0f;
  auto both = [](float x) { return t5::pack2(x, x); };
  const uint64_t x = t5::pack2(fmaxf(x0, -40.0f), fmaxf(x1, -40.0f));
  const uint64_t t = t5::add2(mul2(x, both((float)1.44269504088896340736)), both(shift)), n = t5::add2(t, both(-shift));
  uint64_t r = t5::add2(x, mul2(n, both(-__uint_as_float(0x3F317200u))));
  r = t5::add2(r, mul2(n, both(-(float)(0.69314718055994530942 - 0.693145751953125))));
  uint64_t p = both((float)(1.0 / 5040.0));
  p = t5::add2(mul2(p, r), both((float)(1.0 / 720.0)));
  p = t5::add2(mul2(p, r), both((float)(1.0 / 120.0)));
  p = t5::add2(mul2(p, r), both((float)(1.0 / 24.0)));
  p = t5::add2(mul2(p, r), both((float)(1.0 / 6.0)));
  p = t5::add2(mul2(p, r), both(0.5f));
  p = t5::add2(mul2(p, r), both(1.0f));
  p = t5::add2(mul2(p, r), both(1.0f));
  float p0, p1, t0, t1;
  t5::unpack2(p, p0, p1);
  t5::unpack2(t, t0, t1);
  e0 = __uint_as_float(__float_as_uint(p0) + (__float_as_uint(t0) << 23));
  e1 = __uint_as_float(__float_as_uint(p1) + (__float_as_uint(t1) << 23));
}

template <int C>
__global__ void __launch_bounds__(VF_THREADS, 2) verify_kernel(VerifyArgs a) {
  constexpr int PARTS = C * VF_WARPS, PPL = PARTS / 32;                  // sums of the cluster's warps, per lane
  extern __shared__ __align__(16) uint8_t vf_smem[];
  fa::cluster_arrive();                           // (waited for before the walk)
  MassPair* h1 = reinterpret_cast<MassPair*>(vf_smem);                   // [bucket][copy]: this CTA's masses
  uint64_t* t1 = reinterpret_cast<uint64_t*>(h1 + VF_B1 * VF_COPIES);     // [bucket]: the cluster's
  MassPair* h2 = h1;                                                     // of later rounds
  uint64_t* t2 = t1 + VF_B1;                                             // in turns
  uint32_t* s_list = reinterpret_cast<uint32_t*>(t2 + 2 * VF_B2) + (threadIdx.x >> 5) * VF_KEPT;       // the warp's: columns of weights on their way into a histogram, then the kept words' places
  uint32_t* wt = reinterpret_cast<uint32_t*>(vf_smem + (a.top_p24 < (1u << 24) ? VF_HIST : 0));     // this CTA's weights
  const uint32_t wt_addr = (uint32_t)__cvta_generic_to_shared(wt);
  __shared__ __align__(16) ulonglong2 s_part[2][PARTS];      // what the cluster's warps tell, in turns
  __shared__ uint64_t s_scan[2][VF_WARPS], s_found[2][2];
  __shared__ int s_bin[2];
  __shared__ VerifyNode s_node[VF_NODES];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % C, s = blockIdx.x / C, V = a.V;
  const int c0 = min(V, rank * a.slice), n = min(V, c0 + a.slice) - c0;   // my words [c0, c0 + n)
  const int strip = ((a.slice + VF_THREADS * 4 - 1) / (VF_THREADS * 4) | 1) * 4;      // of a lane: an odd number of 16-byte words (no bank conflicts)
  const int chunk = strip * 32;                   // of a warp
  const int w0 = min(n, warp * chunk), w1 = min(n, w0 + chunk), w4 = w0 + (w1 - w0) / 4 * 4;
  const int l0 = w0 + lane * strip, l1 = w0 < w1 ? min(l0 + strip, (w1 + 3) & ~3) : l0;      // of this lane, where its words are to be consecutive
  int32_t* path = a.path + (int64_t)s * a.max_path;
  float* logp = a.logprobs ? a.logprobs + (int64_t)s * a.max_path : nullptr;

  int row0 = a.offsets[s], rows = a.offsets[s + 1];
  if (row0 < 0 || rows < row0 || rows > a.n_rows) { if (tid == 0) atomicOr(a.status, STATUS_BAD_LENGTH); }
  row0 = min(max(row0, 0), a.n_rows);
  rows = min(max(rows - row0, 0), a.n_rows - row0);
  const bool vec = ((a.logits_stride & 3) == 0) && (((uintptr_t)a.logits & 15) == 0);
  const bool vec_q = ((a.probs_stride & 3) == 0) && (((uintptr_t)a.probs & 15) == 0);
  const bool unit_T = a.temperature == 1.0f, nucleus = a.top_p24 < (1u << 24) && !a.greedy;
  auto scaled = [&](float x) { return unit_T ? x : __fdiv_rn(x, a.temperature); };
  auto fetch = [&](int node) {                    // my words of a node's logits, asynchronously where they are aligned
    const float* row = a.logits + (int64_t)(row0 + node) * a.logits_stride + c0;
    if (vec) for (int i = w0 + lane * 4; i < w4; i += 128) fa::cp_async16(wt_addr + i * 4, row + i);
    fa::cp_commit();
    for (int i = (vec ? w4 : w0) + lane; i < w1; i += 32) wt[i] = __float_as_uint(row[i]);
  };
  if (rows > 0) fetch(0);
  auto gather = [&](int j) {
    VerifyNode v = {a.parents[row0 + j], a.tokens[row0 + j], verify_u24(a.uniform[row0 + j]), 0.f, 0.f};
    if (v.parent >= 0 && v.parent < j && v.token >= 0 && v.token < V) {
      v.logit = a.logits[(int64_t)(row0 + v.parent) * a.logits_stride + v.token];
      if (a.probs) v.q = a.probs[(int64_t)(row0 + v.parent) * a.probs_stride + v.token];
    }
    return v;
  };
  for (int j = tid; j < min(rows, VF_NODES); j += VF_THREADS) s_node[j] = gather(j);
  auto parent_of = [&](int j) { return j < VF_NODES ? s_node[j].parent : a.parents[row0 + j]; };
  auto token_of = [&](int j) { return j < VF_NODES ? s_node[j].token : a.tokens[row0 + j]; };

  int turn = 0, pick = 0;                         // exchanges and selections so far: their shared memory is used in turns
  auto remote = [&](const void* p, int r) { return fa::map_rank((uint32_t)__cvta_generic_to_shared(p), r); };
  auto warp_sum_u64 = [&](uint64_t v) {           // of numbers below 2^50
    return (uint64_t)__reduce_add_sync(0xffffffffu, (uint32_t)v & 0xFFFFFFu) + ((uint64_t)__reduce_add_sync(0xffffffffu, (uint32_t)(v >> 24)) << 24);
  };
  // Every warp tells all CTAs two words; every warp learns, in x[i] and y[i] of lane l, those of part i * 32 + l (parts in
  // order of CTA and warp).  One cluster barrier.
  auto tell = [&](uint64_t x, uint64_t y, uint64_t (&xs)[PPL], uint64_t (&ys)[PPL]) {
    const int b = turn++ & 1;
    if (lane < C) asm volatile("st.shared::cluster.v2.u64 [%0], {%1, %2};" ::"r"(remote(&s_part[b][rank * VF_WARPS + warp], lane)), "l"(x), "l"(y) : "memory");
    fa::cluster_sync();
#pragma unroll
    for (int i = 0; i < PPL; ++i) { const ulonglong2 v = s_part[b][i * 32 + lane]; xs[i] = v.x; ys[i] = v.y; }      // (what is not used is not read)
  };
  auto sum_of = [&](const uint64_t (&xs)[PPL]) {
    uint64_t v = 0;
#pragma unroll
    for (int i = 0; i < PPL; ++i) v += xs[i];
    return warp_sum_u64(v);
  };
  // Adds a bucket's mass to all CTAs' totals (few buckets hold any).
  auto spread = [&](uint64_t* total, MassPair p) {
    const uint64_t m = p.lo + ((uint64_t)p.hi << 16);
    if (m == 0) return;
#pragma unroll
    for (int r = 0; r < C; ++r) asm volatile("red.relaxed.cluster.shared::cluster.add.u64 [%0], %1;" ::"r"(remote(total, r)), "l"(m) : "memory");
  };
  // Among nb <= VF_B2 buckets of masses total[b]: the highest with *above + (mass of the buckets from it on) >= target (the
  // highest that is not empty, for a target of 0).  *above grows by the mass above it.  Leaves zeros behind.
  auto select = [&](uint64_t* total, int nb, uint64_t target, uint64_t* above, uint64_t* at) {
    constexpr int K = VF_B2 / VF_THREADS;
    const int b0 = nb - 1 - tid * K, k = pick++ & 1;
    uint64_t m[K], sum = 0, before = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      m[i] = 0;
      if (b0 - i >= 0) { m[i] = total[b0 - i]; total[b0 - i] = 0; }
      sum += m[i];
    }
    const bool busy = warp * 32 * K < nb;
    if (busy) {
      const uint64_t incl = warp_incl_scan_u64(sum, lane);
      if (lane == 31) s_scan[k][warp] = incl;
      before = incl - sum;
    }
    __syncthreads();
    if (busy) {
      before += warp_sum_u64(lane < warp ? s_scan[k][lane & (VF_WARPS - 1)] : 0);
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const uint64_t run = *above + before;
        if (m[i] > 0 && run + m[i] >= target && (run < target || before == 0)) { s_bin[k] = b0 - i; s_found[k][0] = run; s_found[k][1] = m[i]; }
        before += m[i];
      }
    }
    __syncthreads();
    *above = s_found[k][0]; *at = s_found[k][1];
    return s_bin[k];
  };
  // A lane's column: appends x where w - lo < width, without a branch.  (Reads of the column are volatile, too: they stay behind.)
  const uint32_t column = (uint32_t)__cvta_generic_to_shared(s_list + lane), column_end = column + VF_COLUMN * 128;
  auto append = [&](uint32_t& at, uint32_t w, uint32_t lo, uint32_t width, uint32_t x) {
    asm volatile("{\n .reg .pred p;\n setp.lt.u32 p, %1, %2;\n @p st.shared.u32 [%0], %3;\n @p add.u32 %0, %0, 128;\n}" : "+r"(at) : "r"(w - lo), "r"(width), "r"(x));
  };
  auto listed = [&](int j) { uint32_t x; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(column + j * 128)); return x; };
  // Adds the words of this warp with lo <= w < lo + width to the buckets that bucket(w) gives.  Few words qualify, and a histogram's
  // additions cost a warp the same for one lane as for 32: each lane collects its own first.
  auto histogram = [&](uint32_t lo, uint32_t width, auto bucket) {
    uint32_t at = column;
    auto drain = [&]() {
      const int most = __reduce_max_sync(0xffffffffu, (at - column) >> 7);
      for (int j = 0; j < most; ++j)
        if (column + j * 128 < at) {
          const uint32_t w = listed(j);
          MassPair* p = bucket(w);
          atomicAdd(&p->lo, w & 0xFFFFu);
          atomicAdd(&p->hi, w >> 16);
        }
      at = column;
    };
    auto words = [&](int k) { return l0 + k < l1 ? *reinterpret_cast<const uint4*>(wt + l0 + k) : make_uint4(0, 0, 0, 0); };
    for (int k = 0; k < strip; k += 16) {
      uint4 y[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) y[g] = words(k + 4 * g);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        append(at, y[g].x, lo, width, y[g].x); append(at, y[g].y, lo, width, y[g].y); append(at, y[g].z, lo, width, y[g].z); append(at, y[g].w, lo, width, y[g].w);
        if ((g & 1) && __any_sync(0xffffffffu, at > column_end - 8 * 128)) drain();
      }
    }
    drain();
  };

  if (nucleus) {
    for (int i = tid; i < VF_B1; i += VF_THREADS) t1[i] = 0;
    for (int i = tid; i < 2 * VF_B2; i += VF_THREADS) t2[i] = 0;
  }
  // No CTA writes to another's shared memory before all of the cluster have started.
  fa::cluster_wait();
  __syncthreads();
  int cur = 0, count = 0, next = -1;
  bool live = rows > 0;
  uint64_t xs[PPL], ys[PPL];
  while (live && count < a.max_path) {
    if (rank == 0 && tid == 0) path[count] = cur;
    if (a.eos_id >= 0 && token_of(cur) == a.eos_id) {
      if (rank == 0 && tid == 0 && logp) logp[count] = 0.f;
      ++count;
      break;
    }
    // ---- the first child, whose row is likely to be next
    auto child_behind = [&](int last) {
      for (int j = last + 1; j < rows; j += 32) {
        const unsigned hit = __ballot_sync(0xffffffffu, j + lane < rows && parent_of(j + lane) == cur);
        if (hit) return j + __ffs(hit) - 1;
      }
      return -1;
    };
    int child = count + 1 < a.max_path ? child_behind(cur) : -1;
    // ---- the row's logits are in shared memory: their maximum
    const float* row = a.logits + (int64_t)(row0 + cur) * a.logits_stride;
    fa::cp_wait<0>();
    __syncwarp();
    for (int j = child, k = 0; j >= 0 && k < (C > 8 ? 4 : 1); j = child_behind(j), ++k)      // few sequences: the bandwidth is there
      for (int i = w0 + lane * 32; i < w1; i += 1024)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(a.logits + (int64_t)(row0 + j) * a.logits_stride + c0 + i));
    auto row_max = [&]() {                        // (what is no number counts as excluded)
      float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      for (int i = w0 + lane * 4; i < w4; i += 128) {
        const float4 y = *reinterpret_cast<const float4*>(wt + i);
        m[0] = fmaxf(m[0], y.x); m[1] = fmaxf(m[1], y.y); m[2] = fmaxf(m[2], y.z); m[3] = fmaxf(m[3], y.w);
      }
      if (w4 + lane < w1) m[0] = fmaxf(m[0], __uint_as_float(wt[w4 + lane]));
      tell(__float_as_uint(warp_max(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])))), 0, xs, ys);
      float top = __uint_as_float((uint32_t)xs[0]);
#pragma unroll
      for (int i = 1; i < PPL; ++i) top = fmaxf(top, __uint_as_float((uint32_t)xs[i]));
      return warp_max(top);
    };
    float top = row_max();
    if (top == INFINITY) {                        // too large: excluded too
      for (int i = w0 + lane; i < w1; i += 32) if (__uint_as_float(wt[i]) == INFINITY) wt[i] = __float_as_uint(-INFINITY);
      __syncwarp();
      top = row_max();
    }
    const bool any = top > -INFINITY;
    const float zmax = any ? scaled(top) : 0.f;
    // ---- weights, their sum, and the sum of the exponentials (times 2^30) for the log-probability
    uint64_t tot = 0;
    float sume = 0.f;
    auto weigh = [&](auto unit) {      // (what does not change within a row is decided outside the loop)
      auto z_of = [&](float x) { return radd(unit.value ? x : __fdiv_rn(x, a.temperature), -zmax); };
      for (int i = w0 + lane * 4; i < w4; i += 128) {
        const float4 y = *reinterpret_cast<const float4*>(wt + i);
        float e0, e1, e2, e3;
        verify_exp(z_of(y.x), z_of(y.y), e0, e1);
        verify_exp(z_of(y.z), z_of(y.w), e2, e3);
        const uint4 w = make_uint4(__float2uint_rz(e0), __float2uint_rz(e1), __float2uint_rz(e2), __float2uint_rz(e3));
        sume += (e0 + e1) + (e2 + e3);
        tot += w.x + w.y;                         // (2^31 at most)
        tot += w.z + w.w;
        *reinterpret_cast<uint4*>(wt + i) = w;
      }
      if (w4 + lane < w1) {
        float e, unused;
        verify_exp(z_of(__uint_as_float(wt[w4 + lane])), 0.f, e, unused);
        const uint32_t w = __float2uint_rz(e);
        sume += e; tot += w; wt[w4 + lane] = w;
      }
    };
    if (!any) {
      for (int i = w0 + lane; i < w1; i += 32) wt[i] = 0;
    } else if (a.greedy) {                        // a weight of one at the lowest maximum
      int at = INT_MAX;
      for (int i = w0 + lane; i < w1; i += 32) if (__uint_as_float(wt[i]) == top) at = min(at, c0 + i);
      if (unit_T) weigh(std::true_type()); else weigh(std::false_type());
      tell(__reduce_min_sync(0xffffffffu, at), 0, xs, ys);
      at = INT_MAX;
#pragma unroll
      for (int i = 0; i < PPL; ++i) at = min(at, (int)xs[i]);
      at = __reduce_min_sync(0xffffffffu, at) - c0;
      tot = 0;
      for (int i = w0 + lane; i < w1; i += 32) { wt[i] = i == at; tot += i == at; }
    } else {
      if (unit_T) weigh(std::true_type()); else weigh(std::false_type());
    }
    if (w1 == n && lane < 3 && w1 + lane < ((w1 + 3) & ~3)) wt[w1 + lane] = 0;      // (padding)
    uint64_t left = warp_sum_u64(tot);            // what is left in this warp's words
    // (the warps' sums of exponentials travel as whole multiples of 2^-2 x 2^-30, so that their order plays no part; the sum is 2^30 at least)
    tell(left, (uint64_t)__float2ull_rn(warp_sum(sume) * 4.f), xs, ys);
    uint64_t mass = sum_of(xs);
    const float log_total = logf((float)sum_of(ys) * (1.f / 4294967296.f));
    // ---- the nucleus: the least weight in it and its mass (found when something depends on it)
    uint32_t tau = 1;
    bool whole = !nucleus || mass == 0;           // weights and mass are the nucleus's
    const uint64_t target = mul_shift24(mass, a.top_p24);
    int n_kept = -1;                              // words of this lane in the nucleus, listed in order; -1 in all lanes: any may hold something
    auto find_nucleus = [&]() {
      // Weights below this never decide it: all of them together are at most what it leaves out.
      const uint32_t least = max((uint32_t)((mass - target) / (uint32_t)V), 1u);
      for (int i = tid; i < VF_B1 * VF_COPIES; i += VF_THREADS) h1[i] = MassPair{0, 0};
      __syncthreads();
      // (a weight's leading bits are those of its float, rounded down)
      histogram(least, (1u << 30) + 1 - least, [&](uint32_t w) { return h1 + ((__float_as_uint(__uint2float_rz(w)) >> 20) - (127 << 3)) * VF_COPIES + (lane & (VF_COPIES - 1)); });
      __syncthreads();
      for (int i = tid; i < VF_B1; i += VF_THREADS) {
        MassPair p = {0, 0};                      // (a word sums pieces of 2^18 / C weights below 2^16 at most)
#pragma unroll
        for (int k = 0; k < VF_COPIES; ++k) { const MassPair y = h1[i * VF_COPIES + ((k + i) & (VF_COPIES - 1))]; p.lo += y.lo; p.hi += y.hi; }
        spread(t1 + i, p);
      }
      fa::cluster_sync();
      uint64_t above = 0, at = 0;
      const int b1 = select(t1, VF_B1, target, &above, &at);
      // b1: exponent e and three bits; the bits below in steps of nine
      const int e = b1 >> 3;
      int rest = max(e - 3, 0);
      uint32_t pre = e >= 3 ? 8u | (b1 & 7) : (8u | (b1 & 7)) >> (3 - e);       // the weight's leading bits so far
      for (int round = 0; ; ++round) {
        if (at < (uint64_t)pre << (rest + 1)) { pre = (uint32_t)at; rest = 0; }      // less than two of the bucket's lowest: one weight
        if (rest == 0) break;
        const int bits = min(rest, VF_BITS);
        for (int i = tid; i < VF_B2; i += VF_THREADS) h2[i] = MassPair{0, 0};
        __syncthreads();
        const uint32_t lowest = pre << rest;
        histogram(lowest, 1u << rest, [&](uint32_t w) { return h2 + ((w - lowest) >> (rest - bits)); });
        __syncthreads();
        uint64_t* t = t2 + (round & 1) * VF_B2;
        for (int i = tid; i < VF_B2; i += VF_THREADS) spread(t + i, h2[i]);
        fa::cluster_sync();
        const int bin = select(t, 1 << bits, target, &above, &at);
        pre = (pre << bits) | bin;
        rest -= bits;
      }
      tau = pre;
      mass = above + at;
      whole = true;
      // What is outside becomes 0; few words stay, as a rule: where they are, lane by lane.  (Nobody reads these weights before the
      // next cluster barrier.)
      left = 0;
      uint32_t at_word = column;
      bool full = false;
      for (int i0 = l0; i0 < l1; i0 += 16) {
        uint4 y[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) y[g] = i0 + 4 * g < l1 ? *reinterpret_cast<const uint4*>(wt + i0 + 4 * g) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int i = i0 + 4 * g;
          full = full || at_word > column_end - 4 * 128;
          if (full) at_word = column;
          append(at_word, y[g].x, tau, 0x80000000u, i); append(at_word, y[g].y, tau, 0x80000000u, i + 1);
          append(at_word, y[g].z, tau, 0x80000000u, i + 2); append(at_word, y[g].w, tau, 0x80000000u, i + 3);
          y[g].x = y[g].x >= tau ? y[g].x : 0u; y[g].y = y[g].y >= tau ? y[g].y : 0u; y[g].z = y[g].z >= tau ? y[g].z : 0u; y[g].w = y[g].w >= tau ? y[g].w : 0u;
          left += y[g].x + y[g].y;
          left += y[g].z + y[g].w;
          if (i < l1) *reinterpret_cast<uint4*>(wt + i) = y[g];
        }
      }
      left = warp_sum_u64(left);
      n_kept = __any_sync(0xffffffffu, full) ? -1 : (int)((at_word - column) >> 7);
      __syncwarp();
    };
    // ---- children (every warp by itself, all with the same result)
    int accepted = -1;
    float accepted_logit = 0.f;
    bool lazy = false;                            // a - d with the last test's mass is what is left
    double lazy_mass = 0;
    const float* q = a.probs ? a.probs + (int64_t)(row0 + cur) * a.probs_stride : nullptr;
    auto less = [&](uint32_t w, float prob, double m) -> uint32_t {
      const uint32_t d = __double2uint_rz(verify_scaled(prob, m));         // (the largest number, for more)
      return w > d ? w - d : 0u;
    };
    // What the test with mass m leaves of this warp's words, their sum; `store` puts it in their places.
    auto take = [&](double m, bool store) {
      uint64_t sum = 0;
      if (n_kept >= 0) {
#pragma unroll
        for (int j = 0; j < VF_COLUMN; j += 4) {
          if (!__any_sync(0xffffffffu, j < n_kept)) break;
          int at[4];
          float prob[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) { at[k] = j + k < n_kept ? (int)listed(j + k) : -1; prob[k] = at[k] >= 0 ? q[c0 + at[k]] : 0.f; }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (at[k] < 0) continue;
            const uint32_t x = less(wt[at[k]], prob[k], m);
            sum += x;
            if (store) wt[at[k]] = x;
          }
        }
        return warp_sum_u64(sum);
      }
      constexpr int U = 4;
      for (int i0 = w0 + lane * 4; i0 < w4; i0 += 128 * U) {
        float4 p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + 128 * u;
          if (i >= w4) p[u] = make_float4(0.f, 0.f, 0.f, 0.f);
          else if (vec_q) p[u] = *reinterpret_cast<const float4*>(q + c0 + i);
          else p[u] = make_float4(q[c0 + i], q[c0 + i + 1], q[c0 + i + 2], q[c0 + i + 3]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + 128 * u;
          if (i >= w4) continue;
          uint4 y = *reinterpret_cast<const uint4*>(wt + i);
          y.x = less(y.x, p[u].x, m); y.y = less(y.y, p[u].y, m); y.z = less(y.z, p[u].z, m); y.w = less(y.w, p[u].w, m);
          sum += y.x + y.y;
          sum += y.z + y.w;
          if (store) *reinterpret_cast<uint4*>(wt + i) = y;
        }
      }
      if (w4 + lane < w1) {
        const uint32_t x = less(wt[w4 + lane], q[c0 + w4 + lane], m);
        sum += x;
        if (store) wt[w4 + lane] = x;
      }
      return warp_sum_u64(sum);
    };
    bool refused = false;                         // drafts without probabilities: some child was refused
    bool written = false;                         // weights were written since the last cluster barrier
    auto same_before = [&](int child, int x) {    // has an earlier child the same token?
      bool again = false;
      for (int j = cur + 1; j < child; j += 32) again = again || __any_sync(0xffffffffu, j + lane < child && parent_of(j + lane) == cur && token_of(j + lane) == x);
      return again;
    };
    for (; child >= 0; child = child_behind(child)) {
      if (lazy) { take(lazy_mass, true); lazy = false; written = true; }   // (nobody reads them for that test any more)
      if (written) { fa::cluster_sync(); written = false; }
      const VerifyNode v = child < VF_NODES ? s_node[child] : gather(child);
      const bool in = v.token >= 0 && v.token < V;
      if (!in && tid == 0) atomicOr(a.status, STATUS_BAD_TOKEN);
      if (v.token < 0) continue;                  // no draft: what is left stays
      uint32_t w = 0;
      if (in) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(w) : "r"(remote(wt + v.token % a.slice, v.token / a.slice)) : "memory");
      auto passes = [&]() { return mul_shift24(q ? __double2ull_rz(verify_scaled(v.q, (double)mass)) : mass, v.u24) < w; };
      if (!whole) {
        // The nucleus's mass lies between target and the row's, and a weight is in it when all above it are less than target: a first
        // child that would be accepted at the row's mass, with such a weight, is accepted.  (Most are: no nucleus is needed.)
        if (passes()) {
          bool inside = w > mass - target;
          if (!inside) {
            uint64_t above = 0;
            for (int i = w0 + lane * 4; i < w4; i += 128) {
              const uint4 y = *reinterpret_cast<const uint4*>(wt + i);
              above += (y.x > w ? y.x : 0u) + (y.y > w ? y.y : 0u);
              above += (y.z > w ? y.z : 0u) + (y.w > w ? y.w : 0u);
            }
            if (w4 + lane < w1 && wt[w4 + lane] > w) above += wt[w4 + lane];
            tell(warp_sum_u64(above), 0, xs, ys);
            inside = sum_of(xs) < target;
          }
          if (inside) { accepted = child; accepted_logit = v.logit; break; }
        }
        find_nucleus();
        written = true;
        if (w < tau) w = 0;
      }
      if (!q && same_before(child, v.token)) w = 0;                        // a token that was refused before has nothing left
      if (passes()) { accepted = child; accepted_logit = v.logit; break; }
      if (!q) {
        mass -= w;                                // (all of it is never refused)
        const int i = v.token - c0;
        if (w && i >= w0 && i < w1) left -= w;    // (zeroed below)
        refused = true;
      } else {
        const double m = (double)mass;
        const uint64_t part = take(m, false);
        tell(part, 0, xs, ys);
        written = false;
        const uint64_t all = sum_of(xs);
        if (all) { mass = all; lazy = true; lazy_mass = m; left = part; }
      }
    }
    // ---- without an accepted child: the next token
    if (accepted < 0 && !whole) find_nucleus();
    if (accepted < 0 && mass) {
      tell(left, 0, xs, ys);
      if (refused) {                              // this warp's words of refused tokens, which nobody reads any more
        for (int j = cur + 1 + lane; j < rows; j += 32)
          if (parent_of(j) == cur) { const int x = token_of(j) - c0; if (x >= w0 && x < w1) wt[x] = 0; }
        __syncwarp();
      }
      // mass in the parts before mine
      const uint64_t r = mul_shift24(mass, rows <= VF_NODES ? s_node[0].u24 : verify_u24(a.uniform[row0]));
      uint64_t base = 0;
#pragma unroll
      for (int i = 0; i < PPL; ++i) base += i * 32 + lane < rank * VF_WARPS + warp ? xs[i] : 0;
      base = warp_sum_u64(base);
      if (r >= base && r < base + left) {         // one warp of the cluster
        auto at = [&](int j, uint32_t w) { return lazy && w ? less(w, q[c0 + j], lazy_mass) : w; };
        auto found = [&](int j) {
          const int tok = c0 + j;
          a.next[s] = tok;
          if (logp) logp[count] = radd(scaled(row[tok]), -zmax) - log_total;
        };
        if (n_kept >= 0) {
          uint64_t sum = 0;
          for (int j = 0; j < n_kept; ++j) { const int i = (int)listed(j); sum += at(i, wt[i]); }
          uint64_t run = base + warp_incl_scan_u64(sum, lane) - sum;
          if (r >= run && r < run + sum)
            for (int j = 0; j < n_kept; ++j) {
              const int i = (int)listed(j);
              run += at(i, wt[i]);
              if (run > r) { found(i); break; }
            }
        } else {
          for (int i = w0; i < w1; i += 128) {
            uint32_t x[4];
            uint64_t sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) { const int j = i + lane * 4 + k; x[k] = j < w1 ? at(j, wt[j]) : 0u; sum += x[k]; }
            const uint64_t all = warp_sum_u64(sum);
            if (base + all <= r) { base += all; continue; }
            uint64_t run = base + warp_incl_scan_u64(sum, lane) - sum;
            int tok = -1;
#pragma unroll
            for (int k = 0; k < 4; ++k) { run += x[k]; if (tok < 0 && run > r) tok = i + lane * 4 + k; }
            const unsigned hit = __ballot_sync(0xffffffffu, tok >= 0);
            if (lane == __ffs(hit) - 1) found(tok);
            break;
          }
        }
      }
      next = 0;                                   // written above
    } else if (rank == 0 && tid == 0) {
      if (logp) logp[count] = accepted < 0 ? -INFINITY : radd(scaled(accepted_logit), -zmax) - log_total;
    }
    ++count;
    live = accepted >= 0 && count < a.max_path;
    cur = accepted;
    if (live) {
      fa::cluster_sync();                         // nobody reads this row's weights any more
      fetch(cur);
    }
  }
  fa::cp_wait<0>();
  if (rank == 0) {
    if (tid == 0) { a.n_path[s] = count; if (next < 0) a.next[s] = -1; }
    for (int i = count + tid; i < a.max_path; i += VF_THREADS) { path[i] = -1; if (logp) logp[i] = 0.f; }
  }
  fa::cluster_sync();                             // no CTA leaves while another reads its shared memory
}

}  // namespace rpo
