// Eviction from a paged cache by accumulated attention weight.
//
// Every (sequence, KV head) with more than `budget` tokens keeps exactly `budget` of its slots: first the protected
// ones (position < sinks, or among the `recent` newest positions), then the heaviest; equal weights go to the lower
// slot, a weight that is no number counts least.  A kept slot below `budget` stays where it is; the i-th kept slot at
// or above `budget` (in ascending order) moves into the i-th hole below it.  Attention over cached keys does not
// depend on their order, so only the movers' rows are touched, and since sources lie at or above `budget` and
// destinations below it, all moves are independent and in place.
//
// Selection: one CTA per (sequence, KV head).  The weights' bits are mapped to an unsigned order; a radix select
// (11 + 11 + 10 bits, shared-memory counts) finds the last weight that stays; slot-order prefix sums of ballots
// settle ties, number the holes and pair them with the movers.
#pragma once
#include "paged_kv.cuh"

namespace rpo {

constexpr int EV_THREADS = 1024, EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048;
constexpr int EV_MAX_STRIDE = 1 << 19;      // slots per (sequence, KV head): a kept bit and a hole count per 32 slots in shared memory

struct EvictArgs {
  const int32_t* lens; const float* mass; const int32_t* pos;
  int32_t* lens_out; int32_t* src; float* mass_out; int32_t* pos_out;
  int mass_stride, out_stride, n_seqs, hkv, table_stride, budget, sinks, recent;
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

__host__ __device__ inline size_t evict_smem_bytes(int mass_stride, int budget) {
  return (size_t)((mass_stride + 31) / 32 + (min(budget, mass_stride) + 31) / 32 + 1) * 4;
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(EvictArgs a) {
  extern __shared__ uint32_t ev_smem[];
  __shared__ int hist[EV_BINS];
  __shared__ int s_warp[EV_WARPS], s_warp2[EV_WARPS];
  __shared__ int s_bin, s_above;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sh = blockIdx.x, s = sh / a.hkv;
  const int len = evict_len(a, s);
  int32_t* src = a.src + (int64_t)sh * a.budget;
  if (len <= a.budget) {
    for (int i = tid; i < a.budget; i += EV_THREADS) src[i] = i < len ? i : -1;
    return;
  }
  const float* mass = a.mass + (int64_t)sh * a.mass_stride;
  const int32_t* pos = a.pos + (int64_t)sh * a.mass_stride;
  uint32_t* mask = ev_smem;                                   // kept bit of every slot
  int* holes = (int*)(ev_smem + (a.mass_stride + 31) / 32);    // holes before each 32 slots below the budget

  auto block_max = [&](int v) {
    for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if (lane == 0) s_warp[warp] = v;
    __syncthreads();
    v = s_warp[lane];
    for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  };
  auto block_sum = [&](int v) {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if (lane == 0) s_warp[warp] = v;
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, s_warp[lane]);
  };
  // sum of the lower warps' values
  auto warps_before = [&](int v, int* sh_buf) {
    __syncthreads();
    if (lane == 0) sh_buf[warp] = v;
    __syncthreads();
    return (int)__reduce_add_sync(0xffffffffu, lane < warp ? sh_buf[lane] : 0);
  };

  int newest = INT_MIN;
  for (int i = tid; i < len; i += EV_THREADS) newest = max(newest, pos[i]);
  newest = block_max(newest);
  // positions are 64-bit in the comparison: newest - recent may not fit 32 bits
  auto safe = [&](int p) { return p < a.sinks || (int64_t)p > (int64_t)newest - a.recent; };
  int n_safe = 0;
  for (int i = tid; i < len; i += EV_THREADS) n_safe += safe(pos[i]);
  n_safe = block_sum(n_safe);
  // the class the last kept slot belongs to, and how many of that class stay
  const bool cls = n_safe >= a.budget;
  int need = cls ? a.budget : a.budget - n_safe;

  uint32_t prefix = 0;
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
    __syncthreads();
    for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < len; i += EV_THREADS) {
      if (safe(pos[i]) != cls) continue;
      const uint32_t k = evict_key(mass[i]);
      if (round == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&hist[(k >> shift) & ((1 << bits) - 1)], 1);
    }
    __syncthreads();
    // thread t owns the bins 2047 - 2 t and 2046 - 2 t: counts from the top
    const int hi = EV_BINS - 1 - 2 * tid, c0 = hist[hi], c1 = hist[hi - 1];
    int incl = c0 + c1;
    for (int o = 1; o < 32; o <<= 1) { const int n = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += n; }
    const int before = warps_before(__shfl_sync(0xffffffffu, incl, 31), s_warp) + incl - c0 - c1;
    if (before < need && before + c0 >= need) { s_bin = hi; s_above = before; }
    else if (before + c0 < need && before + c0 + c1 >= need) { s_bin = hi - 1; s_above = before + c0; }
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)s_bin;
    need -= s_above;
  }
  const uint32_t last = prefix;              // slots of the class above `last` stay, and the first `need` equal to it

  const int words = (len + 31) / 32, per = (words + EV_WARPS - 1) / EV_WARPS;
  const int w0 = min(words, warp * per), w1 = min(words, w0 + per);
  int n_eq = 0;
  for (int w = w0; w < w1; ++w) {
    const int i = w * 32 + lane;
    const bool eq = i < len && safe(pos[i]) == cls && evict_key(mass[i]) == last;
    n_eq += __popc(__ballot_sync(0xffffffffu, eq));
  }
  int eq_rank = warps_before(n_eq, s_warp);
  int n_hole = 0, n_mover = 0;
  for (int w = w0; w < w1; ++w) {
    const int i = w * 32 + lane;
    bool kept = false, eq = false;
    if (i < len) {
      const bool sf = safe(pos[i]);
      const uint32_t k = evict_key(mass[i]);
      kept = sf == cls ? k > last : sf;
      eq = sf == cls && k == last;
    }
    const uint32_t eqs = __ballot_sync(0xffffffffu, eq);
    if (eq) kept = eq_rank + __popc(eqs & ((1u << lane) - 1)) < need;
    eq_rank += __popc(eqs);
    const uint32_t m = __ballot_sync(0xffffffffu, kept);
    const uint32_t below = __ballot_sync(0xffffffffu, i < a.budget);
    if (lane == 0) { mask[w] = m; if (below) holes[w] = n_hole; }
    n_hole += __popc(~m & below);
    n_mover += __popc(m & ~below);
  }
  const int hole_base = warps_before(n_hole, s_warp);
  int mover = warps_before(n_mover, s_warp2);
  for (int w = w0 + lane; w < w1; w += 32) if (w * 32 < a.budget) holes[w] += hole_base;
  __syncthreads();
  const int hole_words = (a.budget + 31) / 32;
  for (int w = w0; w < w1; ++w) {
    const int i = w * 32 + lane;
    const uint32_t m = mask[w];
    const bool kept = (m >> lane) & 1;
    if (kept && i < a.budget) src[i] = i;
    const bool moves = kept && i >= a.budget;
    const uint32_t mv = __ballot_sync(0xffffffffu, moves);
    if (moves) {
      const int k = mover + __popc(mv & ((1u << lane) - 1));     // my hole is the k-th
      int lo = 0, hi = hole_words - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (holes[mid] <= k) lo = mid; else hi = mid - 1;
      }
      uint32_t open = ~mask[lo];
      for (int n = k - holes[lo]; n > 0; --n) open &= open - 1;
      src[lo * 32 + __ffs(open) - 1] = i;
    }
    mover += __popc(mv);
  }
}

// Rows, weights and positions of the kept slots to their places; a warp per slot.
template <typename T, int DH>
__global__ void __launch_bounds__(256) evict_move_kernel(PagedView<T> kv, EvictArgs a) {
  constexpr int EPC = 16 / sizeof(T), CPR = DH / EPC;
  const int lane = threadIdx.x & 31, sh = blockIdx.y, s = sh / a.hkv, h = sh % a.hkv;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.lens_out[s] = min(evict_len(a, s), a.budget);
  for (int i = blockIdx.x * 8 + (threadIdx.x >> 5); i < a.budget; i += gridDim.x * 8) {
    const int from = a.src[(int64_t)sh * a.budget + i];
    if (from < 0) continue;
    if (lane == 0) {
      a.mass_out[(int64_t)sh * a.out_stride + i] = a.mass[(int64_t)sh * a.mass_stride + from];
      a.pos_out[(int64_t)sh * a.out_stride + i] = a.pos[(int64_t)sh * a.mass_stride + from];
    }
    if (from == i) continue;
    const int64_t x = paged_row<T, DH>(kv, s, from), y = paged_row<T, DH>(kv, s, i);
    if (x < 0 || y < 0) continue;
    for (int ch = lane; ch < 2 * CPR; ch += 32) {
      T* base = (ch < CPR ? kv.k : kv.v) + h * kv.head_stride + (ch % CPR) * EPC;
      *reinterpret_cast<uint4*>(base + y) = *reinterpret_cast<const uint4*>(base + x);
    }
  }
}

}  // namespace rpo
