// Eviction from a paged cache by accumulated attention weight.
//
// Every (sequence, KV head) with more than `budget` tokens keeps exactly `budget` of its slots: first the protected
// ones (position < sinks, or among the `recent` newest positions), then the heaviest; equal weights go to the lower
// slot, a weight that is no number counts least.  A kept slot below `budget` stays where it is; the i-th kept slot at
// or above `budget` (in ascending order) moves into the i-th hole below it.  Attention over cached keys does not
// depend on their order, so only the movers' rows are touched, and since sources lie at or above `budget` and
// destinations below it, all moves are independent and in place.
//
// One launch does all of it: a CTA, or a cluster of up to eight for long caches, per (sequence, KV head).  Weights are mapped to
// an unsigned order and kept in registers (one read of weights and positions); a radix select (11 + 11 + 10 bits, shared-
// memory counts, added up through the cluster) finds the last weight that stays; prefix sums in slot order settle ties
// and number the holes; holes leave their slots in a shared list that the movers read; the rows are copied
// by all warps, 16 bytes a piece and eight pieces per lane in flight.  Bound by HBM (weights and positions once, moved rows once each way) where much
// moves, by the chain of barriers of the select where little does.  Measured: 512 caches of 1025 slots to 1024 15 us (select and copy as
// two kernels 72), 256 of 1024 .. 6144 to 1024 69 us, four of 65 001 to 8191 56 us (one CTA each and a copy kernel 212).
#pragma once
#include <climits>

#include "attn_tc.cuh"
#include "paged_kv.cuh"

namespace rpo {

constexpr int EV_BINS = 2048;
constexpr int EV_MAX_STRIDE = 1 << 19;      // slots per (sequence, KV head): the longest list of holes that fits shared memory
constexpr int EV_FEW = 4;                   // slots dropped one by one: each costs two barriers, the select costs about twenty
constexpr int EV_MAX_WORDS = 2048;          // kept bits of one CTA's slots, 32 to a word

struct EvictArgs {
  const int32_t* lens; const float* mass; const int32_t* pos;
  int32_t* lens_out; int32_t* src; float* mass_out; int32_t* pos_out;
  int mass_stride, out_stride, n_seqs, hkv, table_stride, budget, sinks, recent;
  uint8_t *k, *v; const int32_t* table; int64_t head_bytes; int row_bytes, n_blocks;
  int write_lens, list_cap;               // list_cap: holes listed per CTA
  int* status;
};

__device__ __forceinline__ int evict_len(const EvictArgs& a, int s) {
  const int n = paged_len(a.lens, s, a.table_stride, a.status);
  if (n > a.mass_stride) { atomicOr(a.status, STATUS_BAD_LENGTH); return a.mass_stride; }
  return n;
}

// Unsigned order of the weights: NaN first, then -inf .. +inf, the two zeros equal.
__device__ __forceinline__ uint32_t evict_key(float x) {
  if (x != x) return 0u;
  const uint32_t b = __float_as_uint(x + 0.0f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__device__ __forceinline__ int64_t evict_row(const EvictArgs& a, int s, int slot) {      // byte offset inside a KV head, or -1
  const int blk = a.table[(int64_t)s * a.table_stride + slot / KV_BLOCK];
  if (blk < 0 || blk >= a.n_blocks) { atomicOr(a.status, STATUS_BAD_BLOCK); return -1; }
  return ((int64_t)blk * KV_BLOCK + slot % KV_BLOCK) * a.row_bytes;
}

__device__ __forceinline__ int ld_cluster_s32(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// KPT slots per thread in registers (0: read again in every pass); a cluster of C CTAs per (sequence, KV head).  Thread
// (warp w, lane) of CTA r owns the slots (r WARPS + w) 32 kpt + 32 k + lane.
template <int THREADS, int KPT, int C>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_kernel(EvictArgs a) {      // 64 registers a thread
  constexpr int WARPS = THREADS / 32, BPT = EV_BINS / THREADS;
  extern __shared__ int ev_list[];                            // slots of the holes this CTA lists
  __shared__ int hist[EV_BINS];
  __shared__ int totals[2][C > 1 ? EV_BINS / C : 1];          // cluster: counts of the bins this CTA owns, of this round and the next
  __shared__ uint32_t mask[KPT ? WARPS * KPT : EV_MAX_WORDS];
  __shared__ int s_warp[2][32], s_cta[2], s_max;
  __shared__ int s_bin, s_above;
  __shared__ uint64_t s_best[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sh = blockIdx.x / C, rank = blockIdx.x % C, s = sh / a.hkv;
  const int len = evict_len(a, s);
  if (a.write_lens && rank == 0 && tid == 0 && sh % a.hkv == 0) a.lens_out[s] = min(len, a.budget);
  int32_t* src = a.src + (int64_t)sh * a.budget;
  const float* mass = a.mass + (int64_t)sh * a.mass_stride;
  const int32_t* pos = a.pos + (int64_t)sh * a.mass_stride;
  float* mass_out = a.mass_out + (int64_t)sh * a.out_stride;
  int32_t* pos_out = a.pos_out + (int64_t)sh * a.out_stride;
  const bool copy_mass = a.mass_out != a.mass, copy_pos = a.pos_out != a.pos;
  if (len <= a.budget) {
    for (int i = rank * THREADS + tid; i < a.budget; i += C * THREADS) {
      src[i] = i < len ? i : -1;
      if (i < len && copy_mass) mass_out[i] = mass[i];
      if (i < len && copy_pos) pos_out[i] = pos[i];
    }
    return;
  }
  const int kpt = (a.mass_stride + C * THREADS - 1) / (C * THREADS);       // at most KPT: the slots are spread over all threads
  const int slot0 = (rank * WARPS + warp) * 32 * kpt + lane;

  auto sync_all = [&]() { if (C > 1) fa::cluster_sync(); else __syncthreads(); };
  auto peer = [&](const void* p, int r) { return fa::map_rank((uint32_t)__cvta_generic_to_shared(p), r); };
  // sum over the warps of this CTA before mine; *all: over the CTA
  auto warps_before = [&](int v, int which, int* all) {
    __syncthreads();
    if (lane == 0) s_warp[which][warp] = v;
    __syncthreads();
    const int w = lane < WARPS ? s_warp[which][lane] : 0;
    *all = (int)__reduce_add_sync(0xffffffffu, w);
    return (int)__reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
  };
  // the same over the slots of the whole cluster, for two counts at once
  auto before2 = [&](int v0, int v1, int* b0, int* b1, int* all1) {
    int t0, t1;
    *b0 = warps_before(v0, 0, &t0);
    *b1 = warps_before(v1, 1, &t1);
    if (C > 1) {
      if (tid == 0) { s_cta[0] = t0; s_cta[1] = t1; }
      fa::cluster_sync();
      const int x0 = lane < C ? ld_cluster_s32(peer(&s_cta[0], lane)) : 0, x1 = lane < C ? ld_cluster_s32(peer(&s_cta[1], lane)) : 0;
      *b0 += (int)__reduce_add_sync(0xffffffffu, lane < rank ? x0 : 0);
      *b1 += (int)__reduce_add_sync(0xffffffffu, lane < rank ? x1 : 0);
      t1 = (int)__reduce_add_sync(0xffffffffu, x1);
      fa::cluster_sync();
    }
    *all1 = t1;
  };

  // ---- weights and positions
  uint32_t key[KPT ? KPT : 1], safe_bits = 0;
  int newest = INT_MIN;
  {
    int p[KPT ? KPT : 1];
    if (KPT) {
#pragma unroll
      for (int k = 0; k < KPT; ++k) {
        const int i = k < kpt ? slot0 + 32 * k : len;
        key[k] = i < len ? evict_key(mass[i]) : 0u;
        p[k] = i < len ? pos[i] : INT_MIN;
        newest = max(newest, p[k]);
      }
    } else {
      for (int k = 0; k < kpt; ++k) if (slot0 + 32 * k < len) newest = max(newest, pos[slot0 + 32 * k]);
    }
    newest = __reduce_max_sync(0xffffffffu, newest);
    if (lane == 0) s_warp[0][warp] = newest;
    __syncthreads();
    newest = __reduce_max_sync(0xffffffffu, lane < WARPS ? s_warp[0][lane] : INT_MIN);
    if (C > 1) {
      if (tid == 0) s_max = newest;
      fa::cluster_sync();
      newest = __reduce_max_sync(0xffffffffu, lane < C ? ld_cluster_s32(peer(&s_max, lane)) : INT_MIN);
    }
    if (KPT)
#pragma unroll
      for (int k = 0; k < KPT; ++k)
        if (k < kpt && slot0 + 32 * k < len && (p[k] < a.sinks || (int64_t)p[k] > (int64_t)newest - a.recent)) safe_bits |= 1u << k;
  }
  auto is_safe = [&](int k) -> bool {                         // (newest - recent may not fit 32 bits)
    if (KPT) return (safe_bits >> k) & 1;
    const int p = pos[slot0 + 32 * k];
    return p < a.sinks || (int64_t)p > (int64_t)newest - a.recent;
  };
  auto get_key = [&](int k) -> uint32_t { return KPT ? key[KPT ? k : 0] : evict_key(mass[slot0 + 32 * k]); };
  auto each = [&](auto f) {                                   // f(k) for my slots that hold a token
    if (KPT) {
#pragma unroll
      for (int k = 0; k < KPT; ++k) if (k < kpt && slot0 + 32 * k < len) f(k);
    } else {
      for (int k = 0; k < kpt; ++k) if (slot0 + 32 * k < len) f(k);
    }
  };
  int n_safe = 0, unused, b0;
  each([&](int k) { n_safe += is_safe(k); });
  n_safe = (int)__reduce_add_sync(0xffffffffu, n_safe);
  before2(0, n_safe, &b0, &unused, &n_safe);
  // the class the last kept slot belongs to, and how many of that class stay
  const bool cls = n_safe >= a.budget;
  int need = cls ? a.budget : a.budget - n_safe;

  // Few slots to drop, none of them protected (a decode step drops one): the lightest, then highest, one after another.
  const int n_drop = len - a.budget;
  const bool few = C == 1 && KPT && n_drop <= EV_FEW && !cls;
  uint32_t last = 0, dropped = 0;                             // dropped: bits of my slots
  if (few) {
    for (int d = 0; d < n_drop; ++d) {
      uint64_t best = ~0ull;
      each([&](int k) {
        if (!((safe_bits | dropped) >> k & 1)) best = min(best, (uint64_t)get_key(k) << 32 | (uint32_t)~(slot0 + 32 * k));
      });
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) best = min(best, (uint64_t)__shfl_xor_sync(0xffffffffu, best, o));
      __syncthreads();
      if (lane == 0) s_best[warp] = best;
      __syncthreads();
      best = lane < WARPS ? s_best[lane] : ~0ull;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) best = min(best, (uint64_t)__shfl_xor_sync(0xffffffffu, best, o));
      const int at = (int)~(uint32_t)best;
      if (at % 32 == lane && at / (32 * kpt) == warp) dropped |= 1u << (at / 32 % kpt);
    }
  } else {
    uint32_t prefix = 0;
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
      for (int i = tid; i < EV_BINS; i += THREADS) hist[i] = 0;
      if (C > 1) for (int i = tid; i < EV_BINS / C; i += THREADS) { totals[(round + 1) & 1][i] = 0; if (round == 0) totals[0][i] = 0; }
      if (C > 1 && round == 0) sync_all(); else __syncthreads();
      each([&](int k) {
        const uint32_t x = get_key(k);
        if (is_safe(k) == cls && (round == 0 || (x >> (shift + bits)) == prefix)) atomicAdd(&hist[(x >> shift) & ((1 << bits) - 1)], 1);
      });
      if (C > 1) {
        // every bin has an owner in the cluster; only bins that hold something are sent there
        __syncthreads();
#pragma unroll
        for (int i = 0; i < BPT; ++i) {
          const int bin = i * THREADS + tid, n = hist[bin];
          if (n) asm volatile("red.relaxed.cluster.shared::cluster.add.s32 [%0], %1;" ::"r"(peer(&totals[round & 1][bin % (EV_BINS / C)], bin / (EV_BINS / C))), "r"(n) : "memory");
        }
      }
      sync_all();
      // thread t owns BPT bins from the top: counts from the top
      int c[BPT], sum = 0;
#pragma unroll
      for (int i = 0; i < BPT; ++i) {
        const int bin = EV_BINS - 1 - tid * BPT - i;
        c[i] = C > 1 ? ld_cluster_s32(peer(&totals[round & 1][bin % (EV_BINS / C)], bin / (EV_BINS / C))) : hist[bin];
        sum += c[i];
      }
      int incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int n = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += n; }
      int above = warps_before(__shfl_sync(0xffffffffu, incl, 31), 0, &unused) + incl - sum;
#pragma unroll
      for (int i = 0; i < BPT; ++i) {
        if (above < need && above + c[i] >= need) { s_bin = EV_BINS - 1 - tid * BPT - i; s_above = above; }
        above += c[i];
      }
      sync_all();                                               // (also: nobody clears counts that others still read)
      prefix = (prefix << bits) | (uint32_t)s_bin;
      need -= s_above;
    }
    last = prefix;                           // slots of the class above `last` stay, and the first `need` equal to it
  }

  // ---- who stays: in slot order
  int n_eq = 0, n_hole = 0, n_mover = 0, eq_rank, hole, mover, n_moves;
#pragma unroll
  for (int k = 0; k < (KPT ? KPT : kpt); ++k) {
    if (k >= kpt) break;
    bool kept = false, eq = false;
    if (slot0 + 32 * k < len) {
      const bool sf = is_safe(k);
      const uint32_t x = get_key(k);
      kept = few ? !(dropped >> k & 1) : sf == cls ? x > last : sf;
      eq = !few && sf == cls && x == last;
    }
    const uint32_t m = __ballot_sync(0xffffffffu, kept), e = __ballot_sync(0xffffffffu, eq);
    if (lane == 0) mask[warp * kpt + k] = m;
    n_eq += __popc(e);                                        // (ties are settled below, when the earlier ones are counted)
  }
  eq_rank = 0;
  if (!few) before2(n_eq, 0, &eq_rank, &b0, &unused);
  else __syncwarp();
#pragma unroll
  for (int k = 0; k < (KPT ? KPT : kpt); ++k) {
    if (k >= kpt) break;
    const bool eq = !few && slot0 + 32 * k < len && is_safe(k) == cls && get_key(k) == last;
    const uint32_t e = __ballot_sync(0xffffffffu, eq);
    const bool take = eq && eq_rank + __popc(e & ((1u << lane) - 1)) < need;
    eq_rank += __popc(e);
    const uint32_t m = mask[warp * kpt + k] | __ballot_sync(0xffffffffu, take);
    __syncwarp();
    if (lane == 0) mask[warp * kpt + k] = m;
    const int i = slot0 + 32 * k;
    n_hole += __popc(__ballot_sync(0xffffffffu, i < a.budget) & ~m);
    n_mover += __popc(__ballot_sync(0xffffffffu, i >= a.budget) & m);
  }
  before2(n_hole, n_mover, &hole, &mover, &n_moves);

  // ---- holes into the list, kept slots below the budget to themselves
  for (int k = 0; k < kpt; ++k) {
    const int i = slot0 + 32 * k;
    const uint32_t m = mask[warp * kpt + k], open = __ballot_sync(0xffffffffu, i < a.budget) & ~m;
    if (i < a.budget) {
      if ((m >> lane) & 1) {
        src[i] = i;
      } else {
        const int nth = hole + __popc(open & ((1u << lane) - 1));
        if (C > 1) {
          const uint32_t at = fa::map_rank((uint32_t)__cvta_generic_to_shared(&ev_list[nth % a.list_cap]), nth / a.list_cap);
          asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(at), "r"(i) : "memory");
        } else ev_list[nth] = i;
      }
    }
    hole += __popc(open);
  }
  sync_all();

  // ---- movers read their hole
  for (int k = 0; k < kpt; ++k) {
    const int i = slot0 + 32 * k;
    const uint32_t m = mask[warp * kpt + k];
    const bool moves = ((m >> lane) & 1) && i >= a.budget;
    const uint32_t mv = __ballot_sync(0xffffffffu, moves);
    if (moves) {
      const int nth = mover + __popc(mv & ((1u << lane) - 1));
      src[C > 1 ? ld_cluster_s32(fa::map_rank((uint32_t)__cvta_generic_to_shared(&ev_list[nth % a.list_cap]), nth / a.list_cap)) : ev_list[nth]] = i;
    }
    mover += __popc(mv);
  }
  sync_all();                                                 // (also: nobody leaves while others read its list)

  // ---- weights, positions and rows to their places: 32 slots per warp and turn.  A lane looks up the pages of one slot;
  // the rows then go in pieces of 16 bytes, eight per lane in flight (4, 8 or 16 slots at once).
  const int row_chunks = a.row_bytes / 16, chunks = 2 * row_chunks, at_once = 256 / chunks;      // K's, then V's
  uint8_t* kb = a.k + (sh % a.hkv) * a.head_bytes;
  uint8_t* vb = a.v + (sh % a.hkv) * a.head_bytes;
  for (int i0 = (rank * WARPS + warp) * 32; i0 < a.budget; i0 += C * THREADS) {
    const int i = i0 + lane, f = i < a.budget ? src[i] : i;
    int64_t from = -1, to = -1;
    if (i < a.budget && (f != i || copy_mass)) mass_out[i] = mass[f];
    if (i < a.budget && (f != i || copy_pos)) pos_out[i] = pos[f];
    if (f != i) { from = evict_row(a, s, f); to = evict_row(a, s, i); }
    if (from < 0) to = -1;
    const uint32_t moved = __ballot_sync(0xffffffffu, to >= 0);
    if (!moved) continue;
    for (int l0 = 0; l0 < 32; l0 += at_once) {
      if (!((moved >> l0) & (at_once == 32 ? 0xffffffffu : (1u << at_once) - 1))) continue;
      uint4 x[8];
      int64_t t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int q = lane + 32 * e, l = l0 + q / chunks, c = q % chunks;
        const int64_t fr = __shfl_sync(0xffffffffu, from, l);
        t[e] = __shfl_sync(0xffffffffu, to, l);
        if (t[e] >= 0) x[e] = *reinterpret_cast<const uint4*>((c < row_chunks ? kb : vb) + fr + (c % row_chunks) * 16);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = (lane + 32 * e) % chunks;
        if (t[e] >= 0) *reinterpret_cast<uint4*>((c < row_chunks ? kb : vb) + t[e] + (c % row_chunks) * 16) = x[e];
      }
    }
  }
}

// Lengths of a call whose output lengths are its input lengths: only when every (sequence, KV head) has read them.
__global__ void __launch_bounds__(256) evict_lens_kernel(EvictArgs a) {
  const int s = blockIdx.x * 256 + threadIdx.x;
  if (s < a.n_seqs) a.lens_out[s] = min(evict_len(a, s), a.budget);
}

}  // namespace rpo
