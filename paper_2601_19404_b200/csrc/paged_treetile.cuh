// Attention of trees of more than 16 rows (nodes x query heads of a KV head) over a caller-owned paged cache, 16-bit storage, on the
// 5th-generation tensor cores.
//
// The items, pieces, pipeline and softmax are those of paged_chunk.cuh, which says why they look as they do; masks come from
// paged_tree.cuh.  What differs: a decode step with drafted tokens has few rows per sequence and many keys, so K and V are read
// for one sub-tile of rows as a rule, and one sub-tile alone is bound by the chain S -> softmax -> P V of its 64-key units (2200
// clocks a unit, 63 % of a copy's rate).  Here both softmax warpgroups and both issuers serve such an item: they take
// alternate units, each with a sum and an output of its own; at the end of a piece warpgroup 0 joins both outputs, which lie in the
// same lanes of tensor memory.  Items of two sub-tiles work as there, one for each warpgroup.  K and V come in rings of 64-key units,
// and both issuers follow every unit's barriers, also those of units that are the other's.
//
// 64 trees of 16 nodes on 1024 .. 6144 tokens, 28 on 4 heads of 128: 121 to 134 us on different cards, with the list of items before
// (7) and the join behind (8); in paged_chunk.cuh's way 136 where it was 123.  Long runs go at a copy's rate (2 trees of 18 nodes on
// three times 40000 .. 60001 tokens: 64 us more for 410 MB more, 6.4 TB/s); what a call costs beyond its bytes is filling and draining
// the rings, 12 units (192 KB) a CTA, and the kernels around.  Steps: one producer for K and V and 8 units 174 (K waits in line behind
// V); two producers 140; 12 units 121 to 129; keys of the next piece sent before its queries, rows of V zeroed by the issuers instead of
// the producer 125 where it was 129.  Not kept: pages prefetched to L2 half a batch ahead, 129 where it was 123; tensor maps
// prefetched, 123.5 where it was 120.7.
// 2 trees of 48 nodes on 40000 .. 60001: 126 to 141 us; their 336 rows are an item of two sub-tiles and one of one, which read the keys
// once each (372 MB instead of 233).  Side by side a unit of the first took 1.17 us and the two units of a tile of the second 1.57, so
// they count 3 and 4 in the list that is cut into shares (126, and 135 where they counted the same, on one card).
#pragma once
#include "paged_chunk.cuh"
#include "paged_tree.cuh"

namespace rpo {

// SINGLE: every item of the call has one sub-tile, so one buffer of queries does and the rings are longer.
template <int DH, bool SINGLE>
struct TreeCfg {
  static constexpr int HALVES = DH / 64, THREADS = 384;
  static constexpr int UNIT = CH_HALF, UNIT_PAGES = UNIT / KV_BLOCK;
  static constexpr int Q_BYTES = CH_BM * DH * 2;                        // one sub-tile
  static constexpr int UNIT_BYTES = UNIT * DH * 2;                      // K or V of a unit
  static constexpr int NS = (SINGLE ? 6 : 5) * (128 / DH);
  static constexpr int JOIN = CH_BM * 8;                                // maximum and sum of the second warpgroup's rows
  static constexpr int BARS = 5 * NS + 16;
  static constexpr int SMEM = (SINGLE ? 1 : 2) * Q_BYTES + 2 * NS * UNIT_BYTES + JOIN + BARS * 8 + 32 + 1024;
};

// Key tiles of an item: the sinks' pages, then the window's, each padded to whole tiles of `pages`.
struct TreeTiles {
  KeyPages kp; int n1, pages;
  __device__ __forceinline__ TreeTiles(const ChunkArgs& c, int p0, int p1, int pages_) : pages(pages_) {
    kp = key_pages(c, p0, p1);
    n1 = (kp.n_first + pages - 1) / pages;
  }
  __device__ __forceinline__ int page0(int t) const { return t < n1 ? t * pages : kp.lo_page + (t - n1) * pages; }
  __device__ __forceinline__ int page_end(int t) const { return t < n1 ? kp.n_first : kp.end_page; }
};

template <int DH, bool SINGLE>
__global__ void __launch_bounds__(TreeCfg<DH, SINGLE>::THREADS, 1)
tree_tile_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                 ChunkTcArgs a) {
  using Cfg = TreeCfg<DH, SINGLE>;
  constexpr int HALVES = Cfg::HALVES, NS = Cfg::NS, UP = Cfg::UNIT_PAGES, PAGE = KV_BLOCK * DH * 2;
  extern __shared__ uint8_t tt_raw[];
  uint8_t* sm = (uint8_t*)(((uintptr_t)tt_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t sQ = tc::smem_u32(sm), sK = sQ + (SINGLE ? 1 : 2) * Cfg::Q_BYTES, sV = sK + NS * Cfg::UNIT_BYTES;
  float2* join_ml = (float2*)(sm + (SINGLE ? 1 : 2) * Cfg::Q_BYTES + 2 * NS * Cfg::UNIT_BYTES);
  uint64_t* bars = (uint64_t*)((uint8_t*)join_ml + Cfg::JOIN);
  uint64_t *k_full = bars, *k_empty = bars + NS, *v_full = bars + 2 * NS, *v_ready = bars + 3 * NS, *v_empty = bars + 4 * NS;
  uint64_t* b2 = bars + 5 * NS;
  uint64_t *s_full = b2, *p_full = b2 + 4;                    // [warpgroup][S buffer]
  uint64_t *pv_done = b2 + 8, *o_full = b2 + 10, *q_full = b2 + 12, *q_free = b2 + 13, *join_full = b2 + 14, *join_free = b2 + 15;
  uint32_t* tmem_slot = (uint32_t*)(bars + Cfg::BARS);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  int* s_first = (int*)(tmem_slot + 2);

  const int warp = (int)t5::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int hkv = a.kv.hkv, rep = a.o.rep;
  const ChunkPlan plan = *a.plan;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      tc::mbar_init(&k_full[i], 1); tc::mbar_init(&k_empty[i], 2);
      tc::mbar_init(&v_full[i], 1); tc::mbar_init(&v_ready[i], 1); tc::mbar_init(&v_empty[i], 2);
    }
    for (int i = 0; i < 4; ++i) { tc::mbar_init(&s_full[i], 1); tc::mbar_init(&p_full[i], 4); }
    for (int i = 0; i < 2; ++i) { tc::mbar_init(&pv_done[i], 1); tc::mbar_init(&o_full[i], 1); }
    tc::mbar_init(q_full, 1); tc::mbar_init(q_free, 2); tc::mbar_init(join_full, 4); tc::mbar_init(join_free, 4);
    *abort_flag = 0; *s_first = 0;
    a.ws.rec[blockIdx.x] = SplitRec{0, 0, 0, 0};
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc::tmem_fence_before();
  __syncthreads();
  tc::tmem_fence_after();
  const uint32_t tmem = *tmem_slot;
  PieceWalkOf<!SINGLE> walk;
  walk.items = a.items; walk.hkv = hkv; walk.over = plan.over;
  walk.f = (int)min((int64_t)plan.total, (int64_t)blockIdx.x * plan.share);
  walk.f_end = (int)min((int64_t)plan.total, (int64_t)(blockIdx.x + 1) * plan.share);
  if (walk.f < walk.f_end)
    for (int i = threadIdx.x; i < plan.n_items; i += Cfg::THREADS) {
      const int2 x = *reinterpret_cast<const int2*>(a.items + i);      // (first, n_tiles)
      if (x.x <= walk.f && walk.f < x.x + (x.y * (SINGLE ? 1 : a.items[i].weight) + plan.over) * hkv) *s_first = i;
    }
  __syncthreads();
  walk.idx = *s_first;
  // Of the current piece: has the item two sub-tiles of rows (a tile is one unit, of both), or one (two units, one for each warpgroup)?
  auto two_of = [&]() { return !SINGLE && walk.it.n_tok > a.tq; };
  auto tiles_of = [&]() { return TreeTiles(a.c, walk.it.key0, walk.it.p0 + walk.it.n_tok - 1, two_of() ? UP : 2 * UP); };

  // Does unit i of the piece hold rows of V that no row of the item sees?  They become zeros first (0 x NaN is not 0).
  auto special = [&](const TreeTiles& tiles, bool two, int i) {
    const int t = walk.t0 + (two ? i : i >> 1), key0 = tiles.page0(t) * KV_BLOCK + (two ? 0 : (i & 1) * Cfg::UNIT), p1 = walk.it.p0 + walk.it.n_tok - 1;
    return t < tiles.n1 ? key0 + Cfg::UNIT > min(a.c.sinks, p1 + 1) : key0 + Cfg::UNIT > walk.it.key0 || key0 < tiles.kp.lo;
  };

  if (warp == 0 || warp == 3) {
    // ------------------------------------------------------------------ producers: warp 0 Q and K, warp 3 V (K runs two own units ahead)
    const bool is_k = warp == 0;
    const uint32_t ring = is_k ? sK : sV;
    uint64_t *full = is_k ? k_full : v_full, *empty = is_k ? k_empty : v_empty;
    bool ok = true;
    int ku = 0;                                              // units sent: ring position
    for (int seg = 0; ok && walk.next(); ++seg) {
      const bool two = two_of();
      const TreeTiles tiles = tiles_of();
      // Lane 0 sends the queries when the last piece's are done with, at the latest before the piece's unit NS: the first NS units only
      // wait for earlier pieces, so that keys are on their way while those finish.
      bool q_sent = !is_k;
      auto send_q = [&](bool now) {
        if (lane != 0 || q_sent || !(now ? tc::mbar_wait(q_free, (seg & 1) ^ 1, abort_flag) : tc::mbar_try_wait(q_free, (seg & 1) ^ 1))) return;
        q_sent = true;
        tc::mbar_expect_tx(q_full, (two ? 2 : 1) * HALVES * rep * a.tq * 128);
        for (int x = 0; x < (two ? 2 : 1); ++x)
          for (int hf = 0; hf < HALVES; ++hf)
            t5::tma_load_3d(sQ + x * Cfg::Q_BYTES + hf * (CH_BM * 128), &q_map, hf * 64, walk.head * rep, walk.it.row0 + x * a.tq, q_full);
      };
      const int32_t* tbl = a.kv.table + (int64_t)walk.it.seq * a.kv.table_stride;
      // The blocks of 32 pages at once, a batch ahead (a unit takes less time than a look-up): lane b holds page b % pages of tile
      // t + b / pages; behind the pages that are seen, the last of them (masked, V zeroed)
      const int batch = 32 / tiles.pages;
      auto lookup = [&](int t) -> int {
        const int tt = t + lane / tiles.pages, b0 = tiles.page0(tt), nv = tiles.page_end(tt) - b0;
        return (tt < walk.t1 && nv > 0) ? tbl[b0 + min(lane % tiles.pages, nv - 1)] : 0;
      };
      int blk = 0, blk_next = lookup(walk.t0);
      for (int t = walk.t0; t < walk.t1 && ok; ++t) {
        const int at = (t - walk.t0) % batch * tiles.pages;            // my tile's first page in the batch
        if (at == 0) {
          blk = blk_next;
          if (t + batch < walk.t1) blk_next = lookup(t + batch);
          if (blk < 0 || blk >= a.kv.n_blocks) { atomicOr(a.kv.status, STATUS_BAD_BLOCK); blk = 0; }
        }
        for (int u = 0; u < (two ? 1 : 2); ++u, ++ku) {
          const int st = ku % NS, b = lane % UP, hf = lane / UP;       // lanes 0 .. UP HALVES - 1: one 16 x 64 box each
          const int y = (walk.head * a.kv.n_blocks + __shfl_sync(0xffffffffu, blk, at + u * UP + b)) * KV_BLOCK;
          send_q((t - walk.t0) * (two ? 1 : 2) + u >= NS);
          if (lane == 0) { ok = tc::mbar_wait(&empty[st], ((ku / NS) & 1) ^ 1, abort_flag); if (ok) tc::mbar_expect_tx(&full[st], Cfg::UNIT_BYTES); }
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) break;
          if (hf < HALVES)
            t5::tma_load_2d(ring + st * Cfg::UNIT_BYTES + (is_k ? hf * (Cfg::UNIT * 128) + b * 2048 : b * PAGE + hf * 2048), is_k ? (const void*)&k_map : (const void*)&v_map,
                            hf * 64, y, &full[st]);
        }
      }
      if (ok) send_q(true);
      ok = __shfl_sync(0xffffffffu, ok && (q_sent || lane != 0), 0);
    }
  } else if (warp < 3) {
    // ------------------------------------------------------------------ MMA issuers: warp 1 for warpgroup 0, warp 2 for warpgroup 1
    constexpr uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(CH_HALF >> 3) << 17) | ((uint32_t)(CH_BM >> 4) << 24);
    constexpr uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((uint32_t)(CH_BM >> 4) << 24);
    const int x = warp - 1;
    const uint32_t dq0 = t5::uniform(t5::desc_lo(sQ, 16)), dk = t5::uniform(t5::desc_lo(sK, 16));
    const uint32_t dv = t5::uniform(t5::desc_lo(sV, 2048)), tm = t5::uniform(tmem);
    const uint32_t t_s = tm + x * CH_BN, t_o = tm + 2 * CH_BN + x * DH;
    bool ok = true;
    int ku = 0, step = 0;                                    // units of the pieces before; units of this warpgroup so far
    uint32_t ready = 0;                                      // bit st: phase of v_ready[st], which special units of two sub-tiles alone complete
    for (int seg = 0; ok && walk.next(); ++seg) {
      const bool two = two_of();
      const TreeTiles tiles = tiles_of();
      const int n_units = (walk.t1 - walk.t0) * (two ? 1 : 2), n_own = walk.t1 - walk.t0, own0 = two ? 0 : x, every = two ? 1 : 2;
      const uint32_t dq = dq0 + (two ? x * (Cfg::Q_BYTES >> 4) : 0);
      const int p1 = walk.it.p0 + walk.it.n_tok - 1, past = walk.it.key0;
      const TreeRow* nodes = a.c.tree + (walk.it.row0 - (walk.it.p0 - past));
      // Zeros for the rows of V in unit i that no row of the item sees (the issuer does it while P is on its way).
      auto zero_unseen = [&](int i, int st) {
        const int t = walk.t0 + (two ? i : i >> 1), key0 = tiles.page0(t) * KV_BLOCK + (two ? 0 : (i & 1) * Cfg::UNIT), seen_end = t < tiles.n1 ? min(a.c.sinks, p1 + 1) : p1 + 1;
        for (int r = lane; r < Cfg::UNIT; r += 32) {
          const int j = key0 + r;
          if (j < seen_end && (j >= tiles.kp.lo || j < a.c.sinks) && !(j >= past && nodes[j - past].depth < 0)) continue;
          const uint32_t row = sV + st * Cfg::UNIT_BYTES + (r >> 4) * PAGE + (r & 15) * 128;
#pragma unroll
          for (int h2 = 0; h2 < HALVES; ++h2)
#pragma unroll
            for (int ch = 0; ch < 8; ++ch) fa::st_zero16(row + h2 * 2048 + ch * 16);
        }
        t5::fence_async_smem();
        __syncwarp();
      };
      int k_at = 0, v_at = 0;                                // units of this piece whose K, V this warp is done with
      // K of the units up to own unit j: the other's are passed on, of mine S = Q K^T is issued.
      auto qk = [&](int j) {
        const int target = own0 + j * every, h = (step + j) & 1;
        for (; k_at <= target; ++k_at) {
          const int st = (ku + k_at) % NS;
          if (!tc::mbar_wait_warp(&k_full[st], ((ku + k_at) / NS) & 1, abort_flag)) return false;
          tc::tmem_fence_after();
          if (t5::elect_one()) {
            if (k_at < target) tc::mbar_arrive(&k_empty[st]);
            else {
              const uint32_t k = dk + st * (Cfg::UNIT_BYTES >> 4);
#pragma unroll
              for (int i = 0; i < DH / 16; ++i)
                t5::umma_ss(t_s + h * CH_HALF, dq + (i >> 2) * (CH_BM * 128 >> 4) + (i & 3) * 2, k + (i >> 2) * (Cfg::UNIT * 128 >> 4) + (i & 3) * 2, idesc_qk, i > 0);
              tc::umma_commit(&s_full[x * 2 + h]);
              tc::umma_commit(&k_empty[st]);
              if (j == n_own - 1) tc::umma_commit(q_free);
            }
          }
        }
        return true;
      };
      ok = tc::mbar_wait_warp(q_full, seg & 1, abort_flag) && qk(0) && (n_own < 2 || qk(1));
      for (int j = 0; j < n_own && ok; ++j) {
        const int target = own0 + j * every, h = (step + j) & 1;
        for (; v_at <= target && ok; ++v_at) {
          const int st = (ku + v_at) % NS;
          const uint32_t ready_parity = (ready >> st) & 1;
          const bool zeros = special(tiles, two, v_at);
          if (zeros && two) ready ^= 1u << st;
          ok = tc::mbar_wait_warp(&v_full[st], ((ku + v_at) / NS) & 1, abort_flag);
          if (!ok) break;
          if (v_at < target) { if (t5::elect_one()) tc::mbar_arrive(&v_empty[st]); continue; }
          if (zeros && (!two || x == 0)) {
            zero_unseen(v_at, st);
            if (two && lane == 0) tc::mbar_arrive(&v_ready[st]);
          } else if (zeros) ok = tc::mbar_wait_warp(&v_ready[st], ready_parity, abort_flag);
          if (!ok) break;
          ok = tc::mbar_wait_warp(&p_full[x * 2 + h], ((step + j) >> 1) & 1, abort_flag);
          if (!ok) break;
          tc::tmem_fence_after();
          if (t5::elect_one()) {
            const uint32_t v = dv + st * (Cfg::UNIT_BYTES >> 4), p = t_s + h * CH_HALF;
#pragma unroll
            for (int b = 0; b < UP; ++b) t5::umma_ts(t_o, p + b * 8, v + b * (PAGE >> 4), idesc_pv, (j > 0 || b > 0) ? 1u : 0u);
            tc::umma_commit(&pv_done[x]);
            tc::umma_commit(&v_empty[st]);
            if (j == n_own - 1) tc::umma_commit(&o_full[x]);
          }
        }
        if (ok && j + 2 < n_own) ok = qk(j + 2);
      }
      for (; ok && k_at < n_units; ++k_at) {                 // the other's last unit
        const int st = (ku + k_at) % NS;
        ok = tc::mbar_wait_warp(&k_full[st], ((ku + k_at) / NS) & 1, abort_flag);
        if (ok && t5::elect_one()) tc::mbar_arrive(&k_empty[st]);
      }
      for (; ok && v_at < n_units; ++v_at) {
        const int st = (ku + v_at) % NS;
        ok = tc::mbar_wait_warp(&v_full[st], ((ku + v_at) / NS) & 1, abort_flag);
        if (ok && t5::elect_one()) tc::mbar_arrive(&v_empty[st]);
      }
      ku += n_units;
      step += n_own;
    }
  } else {
    // ------------------------------------------------------------------ softmax: warps 4..7 warpgroup 0, 8..11 warpgroup 1
    const int x = (warp - 4) >> 2, quad = warp & 3, r = quad * 32 + lane;
    const uint32_t t_s = tmem + ((uint32_t)(quad * 32) << 16) + x * CH_BN;
    const uint32_t t_o = tmem + ((uint32_t)(quad * 32) << 16) + 2 * CH_BN + x * DH;
    const int tok = r / rep;
    uint32_t o_phase = 0;
    int step = 0, joins = 0;                                 // units of this warpgroup so far (phases of its barriers); joins so far
    bool read = true;                                        // warpgroup 1: its last piece's output has been read by the other
    bool ok = true;
    while (ok && walk.next()) {
      const bool two = two_of();
      const int p1 = walk.it.p0 + walk.it.n_tok - 1, past = walk.it.key0, tok0 = two ? x * a.tq : 0;
      const TreeTiles tiles = tiles_of();
      const bool row_valid = tok < a.tq && tok0 + tok < walk.it.n_tok;
      const TreeRow* node = a.c.tree + walk.it.row0 + min(tok0 + tok, walk.it.n_tok - 1);
      const int depth = node->depth, p = past + depth;       // position of the row
      const bool live = row_valid && depth >= 0;
      float m = -INFINITY, l = 0.f;
      bool have_m = false;                                   // every row of the warp has a reference maximum
      for (int t = walk.t0; t < walk.t1; ++t, ++step) {
        const int h = step & 1;
        const uint32_t ts = t_s + h * CH_HALF;
        ok = tc::mbar_wait_warp(&s_full[x * 2 + h], (step >> 1) & 1, abort_flag);
        if (!ok) break;
        tc::tmem_fence_after();
        uint32_t v[CH_HALF];
        tc::tmem_ld32_nowait(ts, v);
        tc::tmem_ld32_nowait(ts + 32, v + 32);
        tc::tmem_ld_wait();
        const int key0 = tiles.page0(t) * KV_BLOCK + (two ? 0 : x * Cfg::UNIT);
        const bool first_range = t < tiles.n1;
        // only cached tokens that every row sees (no row sits behind p1)
        const bool whole = !first_range && key0 + CH_HALF <= past && (a.c.window <= 0 || key0 > p1 - a.c.window);
        bool done = false;
        if (whole && have_m) {
          const float ps = chunk_exp(v, a.scale_log2, m);
          done = __all_sync(0xffffffffu, ps < CH_MOST || !live);
          if (done) l += ps;
          else {
            tc::tmem_ld32_nowait(ts, v);
            tc::tmem_ld32_nowait(ts + 32, v + 32);
            tc::tmem_ld_wait();
          }
        }
        if (!done) {
          if (!whole) {
            const int last = live ? past - 1 : -1, hi = (first_range ? min(last, a.c.sinks - 1) : last) - key0;
            const int lo = a.c.window > 0 ? p - a.c.window + 1 - key0 : -key0, sk = a.c.sinks - key0;
            const uint64_t own = live && !first_range ? tree_bits(node->seen, key0 - past) : 0;
#pragma unroll
            for (int c = 0; c < CH_HALF; ++c) if ((c > hi || (c < lo && c >= sk)) && !((own >> c) & 1)) v[c] = 0xFF800000u;
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < CH_HALF; ++c) mx[c & 3] = fmaxf(mx[c & 3], __uint_as_float(v[c]));
          const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
          const bool move = mt > m;
          if (__any_sync(0xffffffffu, move)) {
            const float factor = move ? (m == -INFINITY ? 0.f : fa::ex2(m - mt)) : 1.f;
            if (t > walk.t0) {
              ok = tc::mbar_wait_warp(&pv_done[x], (step - 1) & 1, abort_flag);      // (at most that one phase is outstanding)
              if (!ok) break;
              tc::tmem_fence_after();
#pragma unroll
              for (int c = 0; c < DH; c += 32) {
                uint32_t w[32];
                tc::tmem_ld32(t_o + c, w);
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * factor);
                t5::tmem_st32_nowait(t_o + c, w);
              }
            }
            if (move) { l *= factor; m = mt; }
            have_m = __all_sync(0xffffffffu, m > -INFINITY || !live);
          }
          l += chunk_exp(v, a.scale_log2, m == -INFINITY ? 0.f : m);
        }
        if (!read) {
          ok = tc::mbar_wait_warp(join_free, (joins - 1) & 1, abort_flag);
          if (!ok) break;
          read = true;
        }
        t5::tmem_st32_nowait(ts, v);
        t5::tmem_st_wait();
        tc::tmem_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&p_full[x * 2 + h]);
      }
      if (!ok) break;
      ok = tc::mbar_wait_warp(&o_full[x], o_phase, abort_flag);
      if (!ok) break;
      o_phase ^= 1;
      tc::tmem_fence_after();
      if (!live) { m = -INFINITY; l = 0.f; }                 // whatever the units without masks gave
      // ---- one sub-tile: warpgroup 0 joins both outputs, which lie in the same lanes of tensor memory
      float f0 = 1.f, f1 = 0.f;
      if (!two) {
        if (x == 1) {
          join_ml[r] = make_float2(m, l);
          tc::tmem_fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(join_full);
          ++joins;
          read = false;
          continue;
        }
        ok = tc::mbar_wait_warp(join_full, joins & 1, abort_flag);
        if (!ok) break;
        ++joins;
        tc::tmem_fence_after();
        const float2 other = join_ml[r];
        const float mm = fmaxf(m, other.x), mu = mm == -INFINITY ? 0.f : mm;
        f0 = fa::ex2(m - mu); f1 = fa::ex2(other.x - mu);
        l = l * f0 + other.y * f1;
        m = mm;
      }
      const bool begins = walk.t0 == 0, ends = walk.t1 == walk.it.n_tiles, split = !(begins && ends);
      const int64_t dst = (int64_t)(walk.it.row0 + tok0 + tok) * a.o.hq + walk.head * rep + r % rep;
      const int64_t part = (int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * a.ws.rows_cap + tok0 * rep + r;
      const float inv = split ? 1.0f : l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
      for (int c = 0; c < DH; c += 32) {
        uint32_t w[32];
        tc::tmem_ld32(t_o + c, w);                          // the whole warp loads, valid rows store
        if (!two) {
          uint32_t y[32];
          tc::tmem_ld32(t_o + DH + c, y);
#pragma unroll
          for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * f0 + __uint_as_float(y[i]) * f1);
        }
        if (!(l > 0.f))                                      // (a row that sees nothing: V that no row sees may have given NaN)
#pragma unroll
          for (int i = 0; i < 32; ++i) w[i] = 0;
        if (row_valid && split) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(a.ws.o + part * DH + c + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        } else if (row_valid) {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            uint4 w4;
            w4.x = fa::pack_bf16(__uint_as_float(w[i]) * inv, __uint_as_float(w[i + 1]) * inv);
            w4.y = fa::pack_bf16(__uint_as_float(w[i + 2]) * inv, __uint_as_float(w[i + 3]) * inv);
            w4.z = fa::pack_bf16(__uint_as_float(w[i + 4]) * inv, __uint_as_float(w[i + 5]) * inv);
            w4.w = fa::pack_bf16(__uint_as_float(w[i + 6]) * inv, __uint_as_float(w[i + 7]) * inv);
            *reinterpret_cast<uint4*>(a.o.out + dst * DH + c + i) = w4;
          }
        }
        __syncwarp();
      }
      tc::tmem_fence_before();
      if (!two) {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(join_free);
      }
      if (row_valid) {
        if (split) a.ws.ml[part] = make_float2(m, l);
        else if (a.o.lse) a.o.lse[dst] = l > 0.f ? m * LN2_F + logf(l) : -INFINITY;
      }
      if (begins && !ends && x == 0 && quad == 2 && lane == 0)
        a.ws.rec[blockIdx.x] = SplitRec{walk.it.row0, walk.head * rep, walk.it.n_tok * rep, walk.parts(plan.share, blockIdx.x)};
    }
  }
  // teardown
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
