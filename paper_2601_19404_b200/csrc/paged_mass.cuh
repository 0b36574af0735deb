// Attention weight that every cached key receives from a chunk of new tokens:
//   mass_out[s][h][j] = mass_in[s][h][j] + sum over rows i of the chunk and query heads of KV head h of
//                       exp(scale q_i . k_j - lse_i)        (keys j that row i sees)
// lse comes from the attention call.  Sums run in a fixed order; nothing is added atomically.  (16-bit storage; the 32-bit
// kernel is in paged_f32.cuh.)
#pragma once
#include "paged_chunk.cuh"
#include "paged_step.cuh"

namespace rpo {

struct MassArgs {
  PagedView<bf16> kv; ChunkArgs c;
  const bf16* q; int64_t q_stride; float scale_log2;
  const float* lse; const float* in; float* out; int stride, rep;
};

// Few rows per sequence (16-bit storage): HBM-bound, K of every page once.  A page's sums need nothing of other pages:
// every warp takes an equal share of the pages of all (sequence, KV head)s, with a ring of pages of its own.  Measured: one
// token for each of 128 sequences of 1024 .. 6144 tokens, 4 KV heads of 128: 87 to 89 us, 5.5 TB/s.
template <int DH, int MT>
struct MassStepCfg {
  static constexpr int STAGES = 3, PAGE_BYTES = KV_BLOCK * DH * 2;
  static constexpr int SMEM = 4 * STAGES * PAGE_BYTES;                 // + (n_seqs + 1) ints
};

template <int DH, int MT>
__global__ void __launch_bounds__(128) mass_step_kernel(MassArgs a) {
  using Cfg = MassStepCfg<DH, MT>;
  constexpr int STAGES = Cfg::STAGES, PB = Cfg::PAGE_BYTES, KS = DH / 16, CPR = DH / 8;
  extern __shared__ __align__(128) uint8_t ms_smem[];
  int* s_pref = reinterpret_cast<int*>(ms_smem + Cfg::SMEM);
  __shared__ int s_scan[4];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, tq = lane & 3;
  const int n_seqs = a.kv.n_seqs, hkv = a.kv.hkv, rep = a.rep;
  // every page of every live key: keys that no row sees are copied
  auto live = [&](int s) { return min(paged_len(a.kv.lens, s, a.kv.table_stride, a.kv.status), a.stride); };
  const int total = page_list<128>(n_seqs, s_pref, s_scan, [&](int s) { return (live(s) + KV_BLOCK - 1) / KV_BLOCK * hkv; });
  const int n_warps = gridDim.x * 4, share = (total + n_warps - 1) / n_warps;
  const int me = blockIdx.x * 4 + warp;
  const int f_end = (int)min((int64_t)total, (int64_t)(me + 1) * share);
  int f = (int)min((int64_t)total, (int64_t)me * share);
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ms_smem) + warp * (STAGES * PB);
  auto sw = [](int row, int chunk) -> uint32_t { return (uint32_t)(row * (DH * 2) + ((chunk ^ (row & 7)) << 4)); };

  while (f < f_end) {
    const int s = page_list_seq(s_pref, n_seqs, f);
    const ChunkSpan sp = chunk_span(a.kv, a.c, s);
    const int n_live = min(sp.len, a.stride), n_pages = (n_live + KV_BLOCK - 1) / KV_BLOCK;
    if (sp.len > a.stride && lane == 0) atomicOr(a.kv.status, STATUS_BAD_LENGTH);
    const int in_seq = f - s_pref[s], h = in_seq / n_pages, i0 = in_seq % n_pages;
    const int n_mine = min(n_pages - i0, f_end - f), R = sp.rows * rep, p0 = sp.len - sp.rows, p1 = sp.len - 1;
    const KeyPages kp = key_pages(a.c, p0, p1);
    const bf16* kb = a.kv.k + h * a.kv.head_stride;
    const int32_t* tbl = a.kv.table + (int64_t)s * a.kv.table_stride;
    uint32_t qf[MT][KS][4];
    int prow[MT][2];
    float lse[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int r = mt * 16 + hh * 8 + g;
        const bool v = r < R;
        const int row = sp.row0 + (v ? r / rep : 0), head = h * rep + (v ? r % rep : 0);
        prow[mt][hh] = v ? p0 + r / rep : -1;                          // a row that does not exist sees nothing
        lse[mt][hh] = v ? a.lse[(int64_t)row * a.c.hq + head] * LOG2E_F : 0.f;
        const uint32_t* qp = reinterpret_cast<const uint32_t*>(a.q + (int64_t)row * a.q_stride + head * DH) + tq;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          qf[mt][k][hh] = v ? qp[k * 8] : 0u;
          qf[mt][k][hh + 2] = v ? qp[k * 8 + 4] : 0u;
        }
      }
    auto seen = [&](int page) { return R > 0 && (page < kp.n_first || (page >= kp.lo_page && page < kp.end_page)); };
    int ids = -1;                                                      // lane t: block of my page 32 b + t
    auto fetch_ids = [&](int base) {
      const int page = i0 + base + lane;
      ids = -1;
      if (base + lane < n_mine && seen(page)) {
        ids = tbl[page];
        if (ids < 0 || ids >= a.kv.n_blocks) { atomicOr(a.kv.status, STATUS_BAD_BLOCK); ids = -1; }
      }
    };
    auto load = [&](int it) {
      const int blk = __shfl_sync(0xffffffffu, ids, it & 31);
      const uint32_t dst = ring + (it % STAGES) * PB;
      if (blk < 0) return;                                             // (not seen, or no block: the scores are not used)
#pragma unroll
      for (int e = 0; e < KV_BLOCK * CPR / 32; ++e) {
        const int x = e * 32 + lane, row = x / CPR, ch = x % CPR;
        fa::cp_async16(dst + sw(row, ch), kb + ((int64_t)blk * KV_BLOCK + row) * DH + ch * 8);
      }
    };
    fetch_ids(0);
    uint32_t have = 0;                                                 // bit it: page `it` of the current 32 was loaded
#pragma unroll
    for (int it = 0; it < STAGES - 1; ++it) { if (it < n_mine) load(it); fa::cp_commit(); }
    have = __ballot_sync(0xffffffffu, ids >= 0);
    uint32_t have_next = 0;
    for (int it = 0; it < n_mine; ++it) {
      if ((it & 31) == 0 && it > 0) have = have_next;
      if (it + STAGES - 1 < n_mine) {
        if (((it + STAGES - 1) & 31) == 0) { fetch_ids(it + STAGES - 1); have_next = __ballot_sync(0xffffffffu, ids >= 0); }
        load(it + STAGES - 1);
      }
      fa::cp_commit();
      const int key0 = (i0 + it) * KV_BLOCK;
      // lane (g < 2, tq) hands over keys 8 g + 2 tq, + 1: what they had is on its way while the scores are computed
      const int j = key0 + g * 8 + tq * 2;
      const int64_t at = ((int64_t)s * hkv + h) * a.stride + j;
      float had0 = 0.f, had1 = 0.f;
      if (a.in && g < 2) {
        if (j < n_live) had0 = a.in[at];
        if (j + 1 < n_live) had1 = a.in[at + 1];
      }
      float w[4] = {0.f, 0.f, 0.f, 0.f};                               // keys 2 tq, 2 tq + 1, and 8 further
      if ((have >> (it & 31)) & 1) {
        fa::cp_wait<STAGES - 1>();
        __syncwarp();
        const uint32_t sk = ring + (it % STAGES) * PB;
        float sc[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int n = 0; n < 2; ++n) sc[mt][n][0] = sc[mt][n][1] = sc[mt][n][2] = sc[mt][n][3] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t b0, b1, b2, b3;
          fa::ldsm_x4(sk + sw(((lane >> 4) << 3) + (lane & 7), k * 2 + ((lane >> 3) & 1)), b0, b1, b2, b3);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) { fa::mma_bf16(sc[mt][0], qf[mt][k], b0, b1); fa::mma_bf16(sc[mt][1], qf[mt][k], b2, b3); }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = fa::ex2(fmaf(sc[mt][e >> 1][2 * hh + (e & 1)], a.scale_log2, -lse[mt][hh]));
              w[e] += chunk_visible(a.c, key0 + (e >> 1) * 8 + tq * 2 + (e & 1), prow[mt][hh]) ? p : 0.f;
            }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] += __shfl_xor_sync(0xffffffffu, w[e], o);
        __syncwarp();
      }
      if (g < 2) {
        if (j < n_live) a.out[at] = had0 + (g ? w[2] : w[0]);
        if (j + 1 < n_live) a.out[at + 1] = had1 + (g ? w[3] : w[1]);
      }
    }
    fa::cp_wait<0>();
    __syncwarp();
    f += n_mine;
  }
}

// Many rows per sequence (16-bit storage) on the 5th-generation tensor cores, with keys and rows swapped against the
// attention: S^T = K Q^T, so that one thread owns one key and sums over the rows in its registers.
//
// An item is 256 keys of one (sequence, KV head), as two sub-tiles of 128 kept in shared memory; the rows of the chunk
// that see any of them stream through in tiles of tq tokens x rep heads <= 128.  All steps of all items form one list,
// cut into equal pieces (one persistent CTA per SM); keys whose rows are spread over several CTAs leave partial sums,
// added up in piece order by mass_merge_kernel.  One exponential per (row, key) bounds it: 16 a clock and SM.  Measured: 8
// chunks of up to 1024 tokens behind 1000 .. 4096, 12 on 2 heads of 128: 83 us with list and join, the exponential unit 82 %
// busy in the steps (94 us while short items counted like long ones in the division of the list).
struct MassItem { int first, steps, seq, key0; int tok0, pad0, pad1, pad2; };      // tok0: first token that sees a key
struct MassWs { float* part; SplitRec* rec; };                                     // part [slot][256]

constexpr int MS_KEYS = 256, MS_ROWS = 128;

__global__ void __launch_bounds__(1024) mass_plan_kernel(PagedView<bf16> kv, ChunkArgs c, int stride, int tq, int n_ctas, int min_share, int over,
                                                         MassItem* items, ChunkPlan* plan) {
  extern __shared__ int pl_first[];                    // items of the sequences before s
  __shared__ int64_t s_warp[32];
  const int tid = threadIdx.x;
  int n_items = 0;
  for (int s0 = 0; s0 < kv.n_seqs; s0 += 1024) {
    const int s = s0 + tid;
    const int n = s < kv.n_seqs ? (min(paged_len(kv.lens, s, kv.table_stride, kv.status), stride) + MS_KEYS - 1) / MS_KEYS : 0;
    int64_t before, all;
    plan_scan(n, before, all, s_warp);
    if (s < kv.n_seqs) pl_first[s] = (int)min((int64_t)OP_MAX_ITEMS, n_items + before);
    if (n_items + all > OP_MAX_ITEMS && tid == 0) atomicOr(kv.status, STATUS_BAD_LENGTH);
    n_items = (int)min((int64_t)OP_MAX_ITEMS, n_items + all);
  }
  __syncthreads();
  int64_t total = 0;
  for (int i0 = 0; i0 < n_items; i0 += 1024) {
    const int i = i0 + tid;
    int64_t n = 0;
    MassItem it = {};
    if (i < n_items) {
      const int s = page_list_seq(pl_first, kv.n_seqs, i);
      const ChunkSpan sp = chunk_span(kv, c, s);
      it.seq = s; it.key0 = (i - pl_first[s]) * MS_KEYS;
      const int p0 = sp.len - sp.rows;
      it.tok0 = max(0, it.key0 - p0);
      int end = sp.rows;
      if (c.window > 0 && it.key0 >= c.sinks) end = (int)min((int64_t)end, (int64_t)it.key0 + MS_KEYS - 1 + c.window - p0);
      it.steps = max(1, (end - it.tok0 + tq - 1) / tq);                // (none: one step in which nothing is seen)
      n = (int64_t)(it.steps + over) * kv.hkv;
      if (sp.len > stride) atomicOr(kv.status, STATUS_BAD_LENGTH);
    }
    int64_t before, all;
    plan_scan(n, before, all, s_warp);
    if (total + all > OP_MAX_TILES) {
      if (tid == 0) atomicOr(kv.status, STATUS_BAD_LENGTH);
      n_items = i0;
      break;
    }
    it.first = (int)(total + before);
    if (i < n_items) items[i] = it;
    total += all;
  }
  if (tid == 0) *plan = ChunkPlan{n_items, (int)total, max(min_share, (int)((total + n_ctas - 1) / n_ctas)), over};
}

template <int DH>
struct MassCfg {
  static constexpr int HALVES = DH / 64;
  static constexpr int K_BYTES = 128 * DH * 2;              // one sub-tile of keys
  static constexpr int Q_BYTES = MS_ROWS * DH * 2;          // one tile of rows
  // An even number of slots: whoever serves every second step then serves the same slots every time and follows their
  // barriers phase by phase (a parity wait says nothing to a waiter two phases behind).
  static constexpr int NSQ = 4;
  static constexpr int SMEM = 2 * K_BYTES + NSQ * Q_BYTES + 1024 + 512 + NSQ * MS_ROWS * 4 + MS_KEYS * 4;
  static constexpr int THREADS = 640;                       // producer, issuer, two warps for the log-sums; four warpgroups of sums
};

struct MassTcArgs {
  PagedView<bf16> kv; ChunkArgs c;
  float scale_log2;
  const float* lse; const float* in; float* out; int stride, rep, tq;
  const MassItem* items; const ChunkPlan* plan; MassWs ws;
};

// Sums of one item over its pieces; 256 threads, one key each.
__global__ void __launch_bounds__(MS_KEYS) mass_merge_kernel(MassWs ws, const float* in, float* out) {
  const SplitRec rec = ws.rec[blockIdx.x];                  // row0: offset of the first key / 2^31 split over two words
  if (rec.n_parts == 0 || (int)threadIdx.x >= rec.rows) return;
  float sum = 0.f;
  for (int p = 0; p < rec.n_parts; ++p) sum += ws.part[(int64_t)(p == 0 ? 2 * blockIdx.x + 1 : 2 * (blockIdx.x + p)) * MS_KEYS + threadIdx.x];
  const int64_t at = ((int64_t)rec.head0 << 31 | (int64_t)rec.row0) + threadIdx.x;
  out[at] = (in ? in[at] : 0.f) + sum;
}

// Sum over the 128 columns (rows of the chunk) of this thread's lane (key) of 2^(s scale - lse); MASKED: columns [lo, hi).
template <bool MASKED>
__device__ __forceinline__ float mass_columns(uint32_t ts, uint32_t ls, float scale_log2, int lo, int hi) {
  const uint64_t sc2 = t5::pack2(scale_log2, scale_log2);
  uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
  for (int c0 = 0; c0 < MS_ROWS; c0 += 32) {
    uint32_t v[32];
    tc::tmem_ld32(ts + c0, v);
#pragma unroll
    for (int c = 0; c < 32; c += 4) {
      uint64_t l01, l23;                                               // two negated log-sums each
      asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(l01), "=l"(l23) : "r"(ls + (c0 + c) * 4));
      float p[4];
      t5::unpack2(t5::fma2(t5::pack2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), sc2, l01), p[0], p[1]);
      t5::unpack2(t5::fma2(t5::pack2(__uint_as_float(v[c + 2]), __uint_as_float(v[c + 3])), sc2, l23), p[2], p[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = fa::ex2(p[e]);
        if (MASKED && (c0 + c + e < lo || c0 + c + e >= hi)) p[e] = 0.f;
      }
      acc[(c >> 1) & 2] = t5::add2(acc[(c >> 1) & 2], t5::pack2(p[0], p[1]));
      acc[((c >> 1) & 2) + 1] = t5::add2(acc[((c >> 1) & 2) + 1], t5::pack2(p[2], p[3]));
    }
  }
  float x, y;
  t5::unpack2(t5::add2(t5::add2(acc[0], acc[1]), t5::add2(acc[2], acc[3])), x, y);
  return x + y;
}

template <int DH>
__global__ void __launch_bounds__(MassCfg<DH>::THREADS, 1)
mass_chunk_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, MassTcArgs a) {
  using Cfg = MassCfg<DH>;
  constexpr int HALVES = Cfg::HALVES, NSQ = Cfg::NSQ;
  extern __shared__ uint8_t mc_raw[];
  uint8_t* sm = (uint8_t*)(((uintptr_t)mc_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t sK = tc::smem_u32(sm), sQ = sK + 2 * Cfg::K_BYTES;
  float* s_lse = (float*)(sm + 2 * Cfg::K_BYTES + NSQ * Cfg::Q_BYTES);       // [NSQ][128], negated, log2 domain
  float* s_sum = s_lse + NSQ * MS_ROWS;                                      // [2][128]: the odd steps' sums
  uint64_t* bars = (uint64_t*)(s_sum + MS_KEYS);
  uint64_t *q_full = bars, *q_empty = bars + NSQ, *l_full = bars + 2 * NSQ;
  uint64_t *s_full = bars + 3 * NSQ, *s_free = s_full + 4, *k_full = s_full + 8, *k_free = s_full + 9;
  uint64_t *x_full = s_full + 10, *x_free = s_full + 12;                     // hand-over of the odd steps' sums, per sub-tile
  uint32_t* tmem_slot = (uint32_t*)(s_full + 14);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  int* s_first = (int*)(tmem_slot + 2);
  const int warp = (int)t5::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, hkv = a.kv.hkv, rep = a.rep, cols = a.tq * rep;
  const ChunkPlan plan = *a.plan;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NSQ; ++i) { tc::mbar_init(&q_full[i], 1); tc::mbar_init(&q_empty[i], 1 + 8); tc::mbar_init(&l_full[i], 1); }
    for (int i = 0; i < 4; ++i) { tc::mbar_init(&s_full[i], 1); tc::mbar_init(&s_free[i], 4); }
    for (int i = 0; i < 2; ++i) { tc::mbar_init(&x_full[i], 4); tc::mbar_init(&x_free[i], 4); }
    tc::mbar_init(k_full, 1); tc::mbar_init(k_free, 1);
    *abort_flag = 0; *s_first = 0;
    a.ws.rec[blockIdx.x] = SplitRec{0, 0, 0, 0};
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a tile behind tq x rep are never filled: zeros, so that no column holds NaN by chance
  for (int i = threadIdx.x; i < NSQ * Cfg::Q_BYTES / 16; i += Cfg::THREADS) fa::st_zero16(sQ + i * 16);
  t5::fence_async_smem();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc::tmem_fence_before();
  __syncthreads();
  tc::tmem_fence_after();
  const uint32_t tmem = *tmem_slot;
  int f = (int)min((int64_t)plan.total, (int64_t)blockIdx.x * plan.share);
  const int f_end = (int)min((int64_t)plan.total, (int64_t)(blockIdx.x + 1) * plan.share);
  if (f < f_end)
    for (int i = threadIdx.x; i < plan.n_items; i += Cfg::THREADS) {
      const int2 x = *reinterpret_cast<const int2*>(a.items + i);
      if (x.x <= f && f < x.x + (x.y + plan.over) * hkv) *s_first = i;
    }
  __syncthreads();
  int idx = *s_first, head = 0, t0 = 0, t1 = 0;
  MassItem it = {};
  auto next = [&]() {                                        // the next piece: every role walks the same ones
    while (f < f_end) {
      it = a.items[idx];
      if (f >= it.first + (it.steps + plan.over) * hkv) it = a.items[++idx];
      const int w = it.steps + plan.over, v0 = (f - it.first) % w, v1 = min(w, v0 + (f_end - f));
      head = (f - it.first) / w;
      t0 = max(0, v0 - plan.over);                           // the first `over` places of an item hold no step
      t1 = v1 - plan.over;
      f += v1 - v0;
      if (t0 < t1) return true;
    }
    return false;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    bool ok = true;
    int qt = 0;
    for (int seg = 0; ok && next(); ++seg) {
      const ChunkSpan sp = chunk_span(a.kv, a.c, it.seq);
      const int live = min(sp.len, a.stride) - it.key0, subs = live > 128 ? 2 : 1;
      if (lane == 0) ok = tc::mbar_wait(k_free, (seg & 1) ^ 1, abort_flag);
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (!ok) break;
      // keys: 8 pages per sub-tile; behind the last page the last one again (those scores are not used).  Pages that
      // no row sees may have no block: page 0 of the pool stands in.
      const int n_pages = (min(live, MS_KEYS) + KV_BLOCK - 1) / KV_BLOCK, page0 = it.key0 / KV_BLOCK;
      const KeyPages kp = key_pages(a.c, sp.len - sp.rows, sp.len - 1);
      const int page = page0 + min(lane & 15, n_pages - 1);
      int blk = 0;
      if (sp.rows > 0 && (page < kp.n_first || (page >= kp.lo_page && page < kp.end_page))) {
        blk = a.kv.table[(int64_t)it.seq * a.kv.table_stride + page];
        if (blk < 0 || blk >= a.kv.n_blocks) { atomicOr(a.kv.status, STATUS_BAD_BLOCK); blk = 0; }
      }
      if (lane == 0) tc::mbar_expect_tx(k_full, subs * Cfg::K_BYTES);
      __syncwarp();
      if ((lane & 15) < subs * 8 && (lane >> 4) < HALVES)
        t5::tma_load_2d(sK + ((lane & 15) >> 3) * Cfg::K_BYTES + (lane >> 4) * (128 * 128) + (lane & 7) * 2048, &k_map, (lane >> 4) * 64,
                        (head * a.kv.n_blocks + blk) * KV_BLOCK, k_full);
      for (int t = t0; t < t1; ++t, ++qt) {
        const int st = qt % NSQ, row = sp.row0 + it.tok0 + t * a.tq;
        if (lane == 0) ok = tc::mbar_wait(&q_empty[st], ((qt / NSQ) & 1) ^ 1, abort_flag);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        if (lane == 0) {
          tc::mbar_expect_tx(&q_full[st], HALVES * cols * 128);
          for (int hf = 0; hf < HALVES; ++hf) t5::tma_load_3d(sQ + st * Cfg::Q_BYTES + hf * (MS_ROWS * 128), &q_map, hf * 64, head * rep, min(row, a.c.n_rows - 1), &q_full[st]);
        }
      }
    }
  } else if (warp == 2 || warp == 3) {
    // ------------------------------------------------------------------ log-sums of the rows: warp 2 even steps, 3 odd ones
    // Columns without a row (their q is zero) get weight 0 from -inf, rows of other chunks are masked later.
    bool ok = true;
    int qt = 0, tok[4], at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const int c = lane + 32 * i; tok[i] = c < cols ? c / rep : 1 << 30; at[i] = c < cols ? c / rep * a.c.hq + c % rep : 0; }
    while (ok && next()) {
      const ChunkSpan sp = chunk_span(a.kv, a.c, it.seq);
      for (int t = t0; t < t1; ++t, ++qt) {
        if ((qt & 1) != (warp & 1)) continue;
        const int st = qt % NSQ, first = it.tok0 + t * a.tq;
        const float* l = a.lse + (int64_t)(sp.row0 + first) * a.c.hq + head * rep;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = tok[i] < sp.rows - first ? l[at[i]] * -LOG2E_F : -INFINITY;
        ok = tc::mbar_wait_warp(&q_empty[st], ((qt / NSQ) & 1) ^ 1, abort_flag);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) s_lse[st * MS_ROWS + lane + 32 * i] = x[i];
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&l_full[st]);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(MS_ROWS >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    const uint32_t dq = t5::uniform(t5::desc_lo(sQ, 16)), dk = t5::uniform(t5::desc_lo(sK, 16)), tm = t5::uniform(tmem);
    bool ok = true;
    int qt = 0;
    uint32_t free_phase = 0;                                 // bit 2 x + b: phase of S buffer b of sub-tile x
    for (int seg = 0; ok && next(); ++seg) {
      const int live = min(paged_len(a.kv.lens, it.seq, a.kv.table_stride, a.kv.status), a.stride) - it.key0, subs = live > 128 ? 2 : 1;
      ok = tc::mbar_wait_warp(k_full, seg & 1, abort_flag);
      if (!ok) break;
      for (int t = t0; t < t1; ++t, ++qt) {
        const int st = qt % NSQ;
        ok = tc::mbar_wait_warp(&q_full[st], (qt / NSQ) & 1, abort_flag);
        if (!ok) break;
        for (int x = 0; x < subs; ++x) {
          const int b = qt & 1;
          ok = tc::mbar_wait_warp(&s_free[x * 2 + b], ((free_phase >> (x * 2 + b)) & 1) ^ 1, abort_flag);
          if (!ok) break;
          free_phase ^= 1u << (x * 2 + b);
          tc::tmem_fence_after();
          if (t5::elect_one()) {
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) {
              const uint32_t off = (i >> 2) * (128 * 128 >> 4) + (i & 3) * 2;
              t5::umma_ss(tm + (x * 2 + b) * 128, dk + x * (Cfg::K_BYTES >> 4) + off, dq + st * (Cfg::Q_BYTES >> 4) + off, idesc, i > 0);
            }
            tc::umma_commit(&s_full[x * 2 + b]);
          }
        }
        if (!ok) break;
        if (t5::elect_one()) { tc::umma_commit(&q_empty[st]); if (t + 1 == t1) tc::umma_commit(k_free); }
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ sums: a warpgroup per (sub-tile x, step parity b)
    // (one warpgroup per sub-tile, two warps per scheduler, left the exponential unit idle for a third of the time)
    const int x = ((warp - 4) >> 2) & 1, b = (warp - 4) >> 3, quad = warp & 3, r = quad * 32 + lane;
    const uint32_t ts = tmem + ((uint32_t)(quad * 32) << 16) + x * 256 + b * 128;
    bool ok = true;
    int qt = 0;
    uint32_t s_phase = 0, x_phase = 0;
    for (int seg = 0; ok && next(); ++seg) {
      const ChunkSpan sp = chunk_span(a.kv, a.c, it.seq);
      const int live = min(sp.len, a.stride) - it.key0, j = it.key0 + x * 128 + r, p0 = sp.len - sp.rows;
      const bool active = x == 0 || live > 128;
      float sum = 0.f;
      for (int t = t0; t < t1; ++t, ++qt) {
        if ((qt & 1) != b) continue;
        const int st = qt % NSQ;
        ok = tc::mbar_wait_warp(&l_full[st], (qt / NSQ) & 1, abort_flag);
        if (ok && active) {
          ok = tc::mbar_wait_warp(&s_full[x * 2 + b], s_phase, abort_flag);
          s_phase ^= 1;
        }
        if (!ok) break;
        if (active) {
          tc::tmem_fence_after();
          const int tok0 = it.tok0 + t * a.tq, n_tok = min(a.tq, sp.rows - tok0), pt = p0 + tok0;
          // of this warp's 32 keys: all seen by all rows of the tile, or none by any?
          const int k_lo = it.key0 + x * 128 + quad * 32, k_hi = k_lo + 31;
          const bool whole = n_tok == a.tq && k_hi <= pt && (a.c.window <= 0 || k_lo > pt + n_tok - 1 - a.c.window || k_hi < a.c.sinks);
          const bool none = k_lo > pt + n_tok - 1 || (a.c.window > 0 && k_hi <= pt - a.c.window && k_lo >= a.c.sinks);
          // columns [lo, hi) of my key
          const int lo = min(max(0, j - pt), MS_ROWS) * rep;
          int end = max(0, n_tok);
          if (a.c.window > 0 && j >= a.c.sinks) end = (int)max((int64_t)0, min((int64_t)end, (int64_t)j + a.c.window - pt));
          const int hi = end * rep;
          const uint32_t ls = tc::smem_u32(s_lse + st * MS_ROWS);
          if (whole) sum += mass_columns<false>(ts, ls, a.scale_log2, 0, 0);
          else if (!none) sum += mass_columns<true>(ts, ls, a.scale_log2, lo, hi);
          tc::tmem_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          if (active) tc::mbar_arrive(&s_free[x * 2 + b]);
          tc::mbar_arrive(&q_empty[st]);
        }
      }
      if (!ok) break;
      // the odd steps' sums join the even ones'
      if (b == 1) {
        ok = tc::mbar_wait_warp(&x_free[x], x_phase ^ 1, abort_flag);
        if (!ok) break;
        s_sum[x * 128 + r] = sum;
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&x_full[x]);
        x_phase ^= 1;
        continue;
      }
      ok = tc::mbar_wait_warp(&x_full[x], x_phase, abort_flag);
      if (!ok) break;
      sum += s_sum[x * 128 + r];
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&x_free[x]);
      x_phase ^= 1;
      const bool begins = t0 == 0, ends = t1 == it.steps;
      const int64_t at = ((int64_t)it.seq * hkv + head) * a.stride + j;
      if (begins && ends) {
        if (x * 128 + r < live) a.out[at] = (a.in ? a.in[at] : 0.f) + sum;
      } else {
        a.ws.part[(int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * MS_KEYS + x * 128 + r] = sum;
        if (begins && x == 0 && quad == 0 && lane == 0)
          a.ws.rec[blockIdx.x] = SplitRec{(int)(at & 0x7FFFFFFF), (int)(at >> 31), min(live, MS_KEYS),
                                          (it.first + (head + 1) * (it.steps + plan.over) - 1) / plan.share - (int)blockIdx.x + 1};
      }
    }
  }
  __syncwarp();
  tc::tmem_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicOr(a.kv.status, STATUS_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(1000000);   // let copies in flight land before the shared memory goes away
    __syncthreads();
  }
  if (warp == 1) {
    tc::tmem_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

}  // namespace rpo
