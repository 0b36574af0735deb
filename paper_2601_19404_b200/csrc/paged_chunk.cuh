// Attention of many rows per sequence over a caller-owned paged cache (16-bit storage) on the 5th-generation tensor
// cores: prompt chunks, tool outputs, turns.
//
// An item is up to 2 tq tokens of one sequence x the rep query heads of one KV head, as two sub-tiles of tq rep <= 128
// packed rows (token-major); its keys come in tiles of 128.  All key tiles of all items form one list, cut into equal
// pieces for one persistent CTA per SM (chunk_prepare_kernel); an item cut by a piece border leaves unnormalised parts that
// split_merge_kernel joins.  A tile is worked on in two halves of 64 keys; per half and sub-tile x:
//
//   S = Q_x K^T      tcgen05.mma, both operands in shared memory (128-byte swizzle, filled by TMA straight from the
//                    pages: 16 x 64 boxes), accumulator in tensor memory, one buffer per half
//   softmax          one warpgroup per sub-tile, one thread per row = TMEM lane: no shuffles, no exchange.  P = 2^(s - m)
//                    goes back to tensor memory as bf16, over the S it came from (the matrix instruction wants both
//                    operands of one type, and V is bf16; a second part of P would be half as much matrix work
//                    again.  Outputs are 2.3e-3 off 64 bits, of which 1.66e-3 is their own rounding)
//   O_x += P V       tcgen05.mma with A = P from tensor memory; accumulates over all tiles.  m is a reference, not
//                    the running maximum.  Halves with masked keys, and all halves until every row of a warp has a
//                    reference, take the maximum and move m (rescaling the row's O in place) where it grows; later
//                    halves take none and move m only where the half's sum exceeds CH_MOST, two per key: the sums
//                    then stay within twice what weights of at most 1 would give (with a bound of 10^12 O left the
//                    range of float32 for values above 3e26).
//
// S of a half is refilled as soon as P V of the same half of the tile before has been issued, so a softmax warp that
// hands over one half finds the next one ready: with 128-key halves (S waits for the softmax of the whole tile before)
// a tile took 4620 clocks, 1900 of them waiting for S.  Rows of V that no row of the item sees (behind the last token,
// between sinks and window) are zeroed in shared memory before P V, since 0 x NaN is not 0; scores there are masked by
// selection.
//
// Measured (28 on 4 heads of 128, 4 x 2048 tokens behind 4096): 600 to 620 us on different cards, 1.0 PFLOP/s.  A half takes about
// 2000 clocks; both sub-tiles' exponentials need 1024 of them, the matrix products 1282 (Q K^T at N = 64 is bound by shared
// memory); neither alone, nor all of tensor and shared memory in use, lets anything run further ahead.  A quarter
// of the exponentials as polynomials on the multiply-add pipe made it 5 % slower.
#pragma once
#include "attn_tc5.cuh"
#include "paged_step.cuh"

namespace rpo {

constexpr int CH_BM = 128, CH_BN = 128;
constexpr int64_t OP_MAX_TILES = ((int64_t)1 << 31) - (1 << 20);
constexpr int CH_HALF = CH_BN / 2;
constexpr float CH_MOST = 2.0f * CH_HALF;      // largest sum of a half's P that is taken without moving the reference

struct ChunkItem { int first, n_tiles, row0, n_tok; int seq, p0, pad0, pad1; };   // p0: position of the item's first token
// `first`, `total`, `share` count (tile, KV head)s, and `over` more for every (item, KV head): what filling the pipeline for
// it and writing its result costs, in tiles, so that CTAs with many short pieces get fewer tiles.
struct ChunkPlan { int n_items, total, share, over; };

// Key tiles of an item: the sinks' pages, then the window's, each padded to whole tiles.
template <int PAGES>
struct KeyTiles {
  KeyPages kp; int n1, n;
  __device__ __forceinline__ KeyTiles(const ChunkArgs& c, int p0, int p1) {
    kp = key_pages(c, p0, p1);
    n1 = (kp.n_first + PAGES - 1) / PAGES;
    n = max(1, n1 + (kp.end_page - kp.lo_page + PAGES - 1) / PAGES);
  }
  __device__ __forceinline__ int page0(int t) const { return t < n1 ? t * PAGES : kp.lo_page + (t - n1) * PAGES; }
  __device__ __forceinline__ int page_end(int t) const { return t < n1 ? kp.n_first : kp.end_page; }
};

// Sum of the lower threads' values, and of all, of a CTA of 1024.
__device__ __forceinline__ void plan_scan(int64_t v, int64_t& before, int64_t& all, int64_t* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int64_t n = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += n; }
  __syncthreads();
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  before = incl - v; all = 0;
  for (int w = 0; w < 32; ++w) { if (w < warp) before += s_warp[w]; all += s_warp[w]; }
}

// What a call needs before its main kernel: CTA 0 sums up the list of items (tok: tokens per item; PAGES: pages per key
// tile), the others write the chunk's K and V to their pages.
template <typename T, int DH, int PAGES>
__global__ void __launch_bounds__(1024) chunk_prepare_kernel(PagedView<T> kv, ChunkArgs c, int tok, int n_ctas, int min_share, int over,
                                                             ChunkItem* items, ChunkPlan* plan, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                             int64_t new_stride) {
  if (blockIdx.x > 0) {
    paged_append<T, DH>(kv, c, k_new, v_new, new_stride, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  extern __shared__ int pl_first[];                    // items of the sequences before s
  __shared__ int64_t s_warp[32];
  const int tid = threadIdx.x;
  // Offsets that go back and forth could name more items than there are rows for: what does not fit is dropped.
  int n_items = 0;
  for (int s0 = 0; s0 < kv.n_seqs; s0 += 1024) {
    const int s = s0 + tid;
    const int n = s < kv.n_seqs ? (chunk_span(kv, c, s).rows + tok - 1) / tok : 0;
    int64_t before, all;
    plan_scan(n, before, all, s_warp);
    if (s < kv.n_seqs) pl_first[s] = (int)min((int64_t)OP_MAX_ITEMS, n_items + before);
    n_items = (int)min((int64_t)OP_MAX_ITEMS, n_items + all);
  }
  __syncthreads();
  int64_t total = 0;
  for (int i0 = 0; i0 < n_items; i0 += 1024) {
    const int i = i0 + tid;
    int64_t n = 0;
    ChunkItem it = {};
    if (i < n_items) {
      const int lo = page_list_seq(pl_first, kv.n_seqs, i);
      const ChunkSpan sp = chunk_span(kv, c, lo);
      const int t0 = (i - pl_first[lo]) * tok;
      it.seq = lo; it.n_tok = min(tok, sp.rows - t0); it.row0 = sp.row0 + t0; it.p0 = sp.len - sp.rows + t0;
      it.n_tiles = KeyTiles<PAGES>(c, it.p0, it.p0 + it.n_tok - 1).n;
      n = (int64_t)(it.n_tiles + over) * kv.hkv;
    }
    int64_t before, all;
    plan_scan(n, before, all, s_warp);
    if (total + all > OP_MAX_TILES) {                    // 2^31 tile x head steps: no call of this size ends in a lifetime
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

// The pieces of one CTA, in order: every role of the CTA walks the same ones.
struct PieceWalk {
  const ChunkItem* items;
  int f, f_end, idx, hkv, over;
  // of the current piece
  ChunkItem it; int head, t0, t1;
  __device__ __forceinline__ bool next() {
    while (f < f_end) {
      it = items[idx];
      if (f >= it.first + (it.n_tiles + over) * hkv) it = items[++idx];  // items hold at least one tile
      const int w = it.n_tiles + over, in_item = f - it.first, v0 = in_item % w, v1 = min(w, v0 + (f_end - f));
      head = in_item / w;
      t0 = max(0, v0 - over);                                        // the first `over` places of an item hold no tile
      t1 = v1 - over;
      f += v1 - v0;
      if (t0 < t1) return true;
    }
    return false;
  }
  // CTAs that work on the current (item, KV head), when it begins in CTA b.
  __device__ __forceinline__ int parts(int share, int b) const { return (it.first + (head + 1) * (it.n_tiles + over) - 1) / share - b + 1; }
};

template <int DH>
struct ChunkCfg {
  static constexpr int HALVES = DH / 64;
  static constexpr int Q_BYTES = CH_BM * DH * 2;            // one sub-tile
  static constexpr int KV_BYTES = CH_BN * DH * 2;           // one K or V tile
  static constexpr int NSK = 2, NSV = 2;
  static constexpr int SMEM = 2 * Q_BYTES + (NSK + NSV) * KV_BYTES + 1024 + 512;      // tiles, alignment, barriers
  static constexpr int THREADS = 384;
};

struct ChunkTcArgs {
  PagedView<bf16> kv; ChunkArgs c;
  float scale_log2;
  AttnOut<bf16> o; SplitWs ws;
  const ChunkItem* items; const ChunkPlan* plan;
  int tq;                                                    // tokens per sub-tile
};

namespace t5 {
// Operand descriptors of these tiles differ in their low word only (address, leading byte offset): the high word
// (stride byte offset 1024, version, 128-byte swizzle) is the same constant, so that loops carry 32-bit values.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t leading_bytes) { return ((addr & 0x3FFFF) >> 4) | ((leading_bytes >> 4) << 16); }
__device__ __forceinline__ void umma_ss(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.b32 p, %4, 0;\n mov.b64 da, {%1, %5};\n mov.b64 db, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}"
      ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(DESC_HI) : "memory");
}
// A from tensor memory (one row per lane, two 16-bit values per column), B from shared memory.
__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 db;\n setp.ne.b32 p, %4, 0;\n mov.b64 db, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}"
      ::"r"(tmem_d), "r"(tmem_a), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(DESC_HI) : "memory");
}
__device__ __forceinline__ void tmem_st32_nowait(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
        "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
        "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// The matrix instructions take their descriptors from uniform registers.  Values that went through a shuffle and code
// under an elected predicate stay there; under `lane == 0` every operand of every instruction is moved across first.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}
// Two float32 values in one 64-bit register: one instruction for both.
__device__ __forceinline__ uint64_t pack2(float x, float y) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y)); return r; }
__device__ __forceinline__ void unpack2(uint64_t r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const void* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_dst), "l"(map), "r"(tc::smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t smem_dst, const void* map, int x, int y, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(smem_dst), "l"(map), "r"(tc::smem_u32(bar)), "r"(x), "r"(y) : "memory");
}
}  // namespace t5

// P = 2^(s scale - m) of one row's half, packed to 16 bits in v[0 .. 31]; returns the sum of the unrounded values.  Two
// scores at a time: packed multiply-add, two exponentials, packed sum.
__device__ __forceinline__ float chunk_exp(uint32_t* v, float scale_log2, float m) {
  const uint64_t sc2 = t5::pack2(scale_log2, scale_log2), mu2 = t5::pack2(-m, -m);
  uint64_t ps[4] = {0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < CH_HALF; c += 2) {
    float p0, p1;
    t5::unpack2(t5::fma2(t5::pack2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), sc2, mu2), p0, p1);
    p0 = fa::ex2(p0); p1 = fa::ex2(p1);
    ps[(c >> 1) & 3] = t5::add2(ps[(c >> 1) & 3], t5::pack2(p0, p1));
    v[c >> 1] = fa::pack_bf16(p0, p1);
  }
  float x0, x1;
  t5::unpack2(t5::add2(t5::add2(ps[0], ps[1]), t5::add2(ps[2], ps[3])), x0, x1);
  return x0 + x1;
}

// tc::mbar_wait_warp with the limit counted from the last tile that passed: while items of one sub-tile pass, however long that
// takes, the second sub-tile's warps already wait for the first S of the next item of two.  (Only there: in every wait
// for S it cost 1.4 % of a long chunk's time.)
__device__ __forceinline__ bool chunk_wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag, const volatile int* passed) {
  bool ok = tc::mbar_try_wait(bar, parity);
  if (!ok) {
    const long long limit = g_wait_limit_cycles;
    long long t0 = clock64();
    int seen = *passed;
    while (!(ok = tc::mbar_try_wait(bar, parity))) {
      if (*abort_flag) break;
      if (clock64() - t0 > limit) {
        const int now = *passed;
        if (now == seen) { *abort_flag = 1; break; }
        seen = now;
        t0 = clock64();
      }
    }
  }
  return __all_sync(0xffffffffu, ok);
}

template <int DH>
__global__ void __launch_bounds__(ChunkCfg<DH>::THREADS, 1)
paged_chunk_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                   ChunkTcArgs a) {
  using Cfg = ChunkCfg<DH>;
  constexpr int HALVES = Cfg::HALVES, NSK = Cfg::NSK, NSV = Cfg::NSV;
  constexpr int PAGE = KV_BLOCK * DH * 2;
  extern __shared__ uint8_t ch_raw[];
  uint8_t* sm = (uint8_t*)(((uintptr_t)ch_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t sQ = tc::smem_u32(sm), sK = sQ + 2 * Cfg::Q_BYTES, sV = sK + NSK * Cfg::KV_BYTES;
  uint64_t* bars = (uint64_t*)(sm + 2 * Cfg::Q_BYTES + (NSK + NSV) * Cfg::KV_BYTES);
  uint64_t *k_full = bars, *k_empty = bars + NSK, *v_full = bars + 2 * NSK, *v_empty = v_full + NSV;
  uint64_t* b2 = v_empty + NSV;
  uint64_t *s_full = b2, *p_full = b2 + 4;                    // [sub-tile][half]
  uint64_t *pv_done = b2 + 8, *o_full = b2 + 10, *q_full = b2 + 12, *q_free = b2 + 13, *v_ready = b2 + 14;
  uint32_t* tmem_slot = (uint32_t*)(v_ready + NSV);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  int* s_first = (int*)(tmem_slot + 2);
  volatile int* s_passed = (volatile int*)(tmem_slot + 3);   // the last tile without work for the second sub-tile

  const int warp = (int)t5::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int hkv = a.kv.hkv, rep = a.o.rep;
  const ChunkPlan plan = *a.plan;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NSK; ++i) { tc::mbar_init(&k_full[i], 1); tc::mbar_init(&k_empty[i], 2); }
    for (int i = 0; i < NSV; ++i) { tc::mbar_init(&v_full[i], 1); tc::mbar_init(&v_ready[i], 1); tc::mbar_init(&v_empty[i], 2); }
    for (int i = 0; i < 4; ++i) { tc::mbar_init(&s_full[i], 1); tc::mbar_init(&p_full[i], 4); }
    for (int i = 0; i < 2; ++i) { tc::mbar_init(&pv_done[i], 1); tc::mbar_init(&o_full[i], 1); }
    tc::mbar_init(q_full, 1); tc::mbar_init(q_free, 2);
    *abort_flag = 0; *s_first = 0; *s_passed = 0;
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
  PieceWalk walk;
  walk.items = a.items; walk.hkv = hkv; walk.over = plan.over;
  walk.f = (int)min((int64_t)plan.total, (int64_t)blockIdx.x * plan.share);
  walk.f_end = (int)min((int64_t)plan.total, (int64_t)(blockIdx.x + 1) * plan.share);
  if (walk.f < walk.f_end)
    for (int i = threadIdx.x; i < plan.n_items; i += Cfg::THREADS) {
      const int2 x = *reinterpret_cast<const int2*>(a.items + i);      // (first, n_tiles)
      if (x.x <= walk.f && walk.f < x.x + (x.y + plan.over) * hkv) *s_first = i;
    }
  __syncthreads();
  walk.idx = *s_first;

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    bool ok = true;
    int kt = 0;                                              // tiles sent: ring position of K and V
    for (int seg = 0; ok && walk.next(); ++seg) {
      const KeyTiles<CH_BN / KV_BLOCK> kt_of(a.c, walk.it.p0, walk.it.p0 + walk.it.n_tok - 1);
      const bool two = walk.it.n_tok > a.tq;
      if (lane == 0) ok = tc::mbar_wait(q_free, (seg & 1) ^ 1, abort_flag);
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (!ok) break;
      if (lane == 0) {
        tc::mbar_expect_tx(q_full, (two ? 2 : 1) * HALVES * rep * a.tq * 128);
        for (int x = 0; x < (two ? 2 : 1); ++x)
          for (int hf = 0; hf < HALVES; ++hf)
            t5::tma_load_3d(sQ + x * Cfg::Q_BYTES + hf * (CH_BM * 128), &q_map, hf * 64, walk.head * rep, walk.it.row0 + x * a.tq, q_full);
      }
      const int32_t* tbl = a.kv.table + (int64_t)walk.it.seq * a.kv.table_stride;
      // lane b < 8: block of page b of tile t; behind the pages that are seen, the last of them (masked, V zeroed)
      auto lookup = [&](int t) -> int {
        const int b0 = kt_of.page0(t), nv = kt_of.page_end(t) - b0;
        return (lane < CH_BN / KV_BLOCK && nv > 0) ? tbl[b0 + min(lane, nv - 1)] : 0;
      };
      int blk_next = lookup(walk.t0);
      for (int t = walk.t0; t < walk.t1; ++t, ++kt) {
        int blk = blk_next;
        if (t + 1 < walk.t1) blk_next = lookup(t + 1);
        if (blk < 0 || blk >= a.kv.n_blocks) { atomicOr(a.kv.status, STATUS_BAD_BLOCK); blk = 0; }
        const int sk = kt % NSK, sv = kt % NSV;
        const int b = lane & 7, hf = lane >> 3;              // lanes 0 .. 8 HALVES - 1: one 16 x 64 box each
        const int y = (walk.head * a.kv.n_blocks + __shfl_sync(0xffffffffu, blk, b)) * KV_BLOCK;
        if (lane == 0) { ok = tc::mbar_wait(&k_empty[sk], ((kt / NSK) & 1) ^ 1, abort_flag); if (ok) tc::mbar_expect_tx(&k_full[sk], Cfg::KV_BYTES); }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        if (hf < HALVES) t5::tma_load_2d(sK + sk * Cfg::KV_BYTES + hf * (CH_BN * 128) + b * 2048, &k_map, hf * 64, y, &k_full[sk]);
        if (lane == 0) { ok = tc::mbar_wait(&v_empty[sv], ((kt / NSV) & 1) ^ 1, abort_flag); if (ok) tc::mbar_expect_tx(&v_full[sv], Cfg::KV_BYTES); }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        if (hf < HALVES) t5::tma_load_2d(sV + sv * Cfg::KV_BYTES + b * PAGE + hf * 2048, &v_map, hf * 64, y, &v_full[sv]);
      }
    }
  } else if (warp == 3) {
    // ------------------------------------------------------------------ rows of V that no row of the item sees: zeros
    bool ok = true;
    int kt = 0;
    while (ok && walk.next()) {
      const int p1 = walk.it.p0 + walk.it.n_tok - 1;
      const KeyTiles<CH_BN / KV_BLOCK> kt_of(a.c, walk.it.p0, p1);
      for (int t = walk.t0; t < walk.t1; ++t, ++kt) {
        const int sv = kt % NSV;
        ok = tc::mbar_wait_warp(&v_full[sv], (kt / NSV) & 1, abort_flag);
        if (!ok) break;
        const int key0 = kt_of.page0(t) * KV_BLOCK, seen_end = t < kt_of.n1 ? min(a.c.sinks, p1 + 1) : p1 + 1;
        if (key0 + CH_BN > seen_end || (t >= kt_of.n1 && key0 < kt_of.kp.lo)) {
          for (int r = lane; r < CH_BN; r += 32) {
            const int j = key0 + r;
            if (j < seen_end && (j >= kt_of.kp.lo || j < a.c.sinks)) continue;
            const uint32_t at = sV + sv * Cfg::KV_BYTES + (r >> 4) * PAGE + (r & 15) * 128;
#pragma unroll
            for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
              for (int ch = 0; ch < 8; ++ch) fa::st_zero16(at + hf * 2048 + ch * 16);
          }
          t5::fence_async_smem();
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&v_ready[sv]);
      }
    }
  } else if (warp < 3) {
    // ------------------------------------------------------------------ MMA issuers: warp 1 sub-tile 0, warp 2 sub-tile 1
    // (One issuer for both left the tensor pipe idle between its waits: an instruction of 64 clocks occupies the thread
    // that issues it for as long.  Each warp waits together, one lane issues.)
    constexpr uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(CH_HALF >> 3) << 17) | ((uint32_t)(CH_BM >> 4) << 24);
    constexpr uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((uint32_t)(CH_BM >> 4) << 24);
    const int x = warp - 1;
    const uint32_t dq = t5::uniform(t5::desc_lo(sQ + x * Cfg::Q_BYTES, 16)), dk = t5::uniform(t5::desc_lo(sK, 16));
    const uint32_t dv = t5::uniform(t5::desc_lo(sV, 2048)), tm = t5::uniform(tmem);
    const uint32_t t_s = tm + x * CH_BN, t_o = tm + 2 * CH_BN + x * DH;
    bool ok = true;
    int kt = 0;
    uint32_t p_phase = 0;
    auto issue_qk = [&](int h, int sk) {
      const uint32_t k = dk + sk * (Cfg::KV_BYTES >> 4) + h * (CH_HALF * 128 >> 4);
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) {
        const uint32_t off = (i >> 2) * (CH_BN * 128 >> 4) + (i & 3) * 2;
        t5::umma_ss(t_s + h * CH_HALF, dq + off, k + off, idesc_qk, i > 0);
      }
      tc::umma_commit(&s_full[x * 2 + h]);
    };
    auto issue_pv = [&](int h, int sv, bool first) {
      const uint32_t v = dv + sv * (Cfg::KV_BYTES >> 4) + h * (CH_HALF / KV_BLOCK * PAGE >> 4), p = t_s + h * CH_HALF;
#pragma unroll
      for (int b = 0; b < CH_HALF / KV_BLOCK; ++b) t5::umma_ts(t_o, p + b * 8, v + b * (PAGE >> 4), idesc_pv, (!first || b > 0) ? 1u : 0u);
      tc::umma_commit(&pv_done[x]);
    };
    for (int seg = 0; ok && walk.next(); ++seg) {
      const bool idle = x == 1 && walk.it.n_tok <= a.tq;                 // no second sub-tile: only release what the first uses
      ok = tc::mbar_wait_warp(q_full, seg & 1, abort_flag) && tc::mbar_wait_warp(&k_full[kt % NSK], (kt / NSK) & 1, abort_flag);
      if (!ok) break;
      tc::tmem_fence_after();
      if (t5::elect_one()) {
        if (idle) {
          tc::mbar_arrive(&k_empty[kt % NSK]);
          tc::mbar_arrive(q_free);
        } else {
          issue_qk(0, kt % NSK);
          issue_qk(1, kt % NSK);
          tc::umma_commit(&k_empty[kt % NSK]);
          if (walk.t1 - walk.t0 == 1) tc::umma_commit(q_free);
        }
      }
      for (int t = walk.t0; t < walk.t1 && ok; ++t, ++kt) {
        const int sv = kt % NSV, sk = (kt + 1) % NSK;
        const bool more = t + 1 < walk.t1;
        ok = tc::mbar_wait_warp(&v_ready[sv], (kt / NSV) & 1, abort_flag);
        if (ok && more) ok = tc::mbar_wait_warp(&k_full[sk], ((kt + 1) / NSK) & 1, abort_flag);
        if (!ok) break;
        if (idle) {
          if (t5::elect_one()) {
            tc::mbar_arrive(&v_empty[sv]);
            if (more) tc::mbar_arrive(&k_empty[sk]);
            *s_passed = kt + 1;
          }
          continue;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          ok = tc::mbar_wait_warp(&p_full[x * 2 + h], p_phase, abort_flag);
          if (!ok) break;
          tc::tmem_fence_after();
          if (t5::elect_one()) {
            issue_pv(h, sv, t == walk.t0 && h == 0);
            if (more) issue_qk(h, sk);
            if (h == 1) {
              tc::umma_commit(&v_empty[sv]);
              if (more) tc::umma_commit(&k_empty[sk]);
              else tc::umma_commit(&o_full[x]);
              if (t + 2 == walk.t1) tc::umma_commit(q_free);
            }
          }
        }
        p_phase ^= 1;
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ softmax: warps 4..7 sub-tile 0, 8..11 sub-tile 1
    const int x = (warp - 4) >> 2, quad = warp & 3, r = quad * 32 + lane;
    const uint32_t t_s = tmem + ((uint32_t)(quad * 32) << 16) + x * CH_BN;
    const uint32_t t_o = tmem + ((uint32_t)(quad * 32) << 16) + 2 * CH_BN + x * DH;
    const int tok = r / rep;
    const bool in_tile = tok < a.tq;
    uint32_t s_phase = 0, o_phase = 0;
    int steps = 0;                                           // halves of this sub-tile so far: phases of pv_done
    bool ok = true, skipped = false;
    while (ok && walk.next()) {
      if (x == 1 && walk.it.n_tok <= a.tq) { skipped = true; continue; }
      if (skipped) {
        ok = chunk_wait_warp(&s_full[2], s_phase, abort_flag, s_passed);     // (x is 1; the first half's S)
        if (!ok) break;
        skipped = false;
      }
      const int p_item = walk.it.p0, p1 = p_item + walk.it.n_tok - 1;
      const KeyTiles<CH_BN / KV_BLOCK> kt_of(a.c, p_item, p1);
      const bool row_valid = in_tile && x * a.tq + tok < walk.it.n_tok;
      const int p_lo = p_item + x * a.tq, p_hi = min(p1, p_lo + a.tq - 1);     // positions of my sub-tile
      const int p = min(p_lo + tok, p_hi);
      float m = -INFINITY, l = 0.f;
      bool have_m = false;                                   // every row of the warp has a reference maximum
      // Halves [u_whole0, u_whole1) hold only keys that every row of the sub-tile sees (of the window's tiles; halves of
      // the sinks' tiles are masked one by one).
      const int first_key = kt_of.page0(kt_of.n1) * KV_BLOCK;
      const int from = a.c.window > 0 ? max(0, p_hi - a.c.window + 1 - first_key) : 0;
      const int u_whole0 = 2 * kt_of.n1 + (from + CH_HALF - 1) / CH_HALF;
      const int u_whole1 = 2 * kt_of.n1 + max(0, p_lo + 1 - first_key) / CH_HALF;
      for (int u = 2 * walk.t0; u < 2 * walk.t1; ++u, ++steps) {
        const int h = u & 1;
        const uint32_t ts = t_s + h * CH_HALF;
        ok = tc::mbar_wait_warp(&s_full[x * 2 + h], s_phase, abort_flag);
        if (!ok) break;
        if (h == 1) s_phase ^= 1;
        tc::tmem_fence_after();
        uint32_t v[CH_HALF];
        tc::tmem_ld32_nowait(ts, v);
        tc::tmem_ld32_nowait(ts + 32, v + 32);
        tc::tmem_ld_wait();
        const bool whole = u >= u_whole0 && u < u_whole1;
        // All keys seen and every row has a reference: no maximum is needed, any reference is exact as long as nothing
        // overflows, and the half's sum tells.  (S stays in tensor memory until P is stored over it.)
        bool done = false;
        if (whole && have_m) {
          const float ps = chunk_exp(v, a.scale_log2, m);
          done = __all_sync(0xffffffffu, ps < CH_MOST || !row_valid);
          if (done) l += ps;
          else {
            tc::tmem_ld32_nowait(ts, v);
            tc::tmem_ld32_nowait(ts + 32, v + 32);
            tc::tmem_ld_wait();
          }
        }
        if (!done) {
          if (!whole) {
            const int key0 = kt_of.page0(u >> 1) * KV_BLOCK + h * CH_HALF;
            const bool first_range = (u >> 1) < kt_of.n1;
            const int hi = (first_range ? min(p, a.c.sinks - 1) : p) - key0;
            const int lo = a.c.window > 0 ? p - a.c.window + 1 - key0 : -key0, sk = a.c.sinks - key0;
#pragma unroll
            for (int c = 0; c < CH_HALF; ++c) if (c > hi || (c < lo && c >= sk)) v[c] = 0xFF800000u;
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < CH_HALF; ++c) mx[c & 3] = fmaxf(mx[c & 3], __uint_as_float(v[c]));
          const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
          const bool move = mt > m;
          if (__any_sync(0xffffffffu, move)) {
            const float factor = move ? (m == -INFINITY ? 0.f : fa::ex2(m - mt)) : 1.f;
            if (u > 2 * walk.t0) {
              // O is at rest once P V of the half before is done.  (This half's S was issued behind the P V of two
              // halves ago, so at most that one phase is outstanding and its parity cannot be taken for an older one.)
              ok = tc::mbar_wait_warp(&pv_done[x], (steps - 1) & 1, abort_flag);
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
            have_m = __all_sync(0xffffffffu, m > -INFINITY || !row_valid);
          }
          l += chunk_exp(v, a.scale_log2, m == -INFINITY ? 0.f : m);
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
      const bool begins = walk.t0 == 0, ends = walk.t1 == walk.it.n_tiles, split = !(begins && ends);
      const float inv = l > 0.f ? 1.0f / l : 0.f;
      const int64_t dst = (int64_t)(walk.it.row0 + x * a.tq + tok) * a.o.hq + walk.head * rep + r % rep;
      const int64_t part = (int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * a.ws.rows_cap + x * (a.tq * rep) + r;
#pragma unroll
      for (int c = 0; c < DH; c += 32) {
        uint32_t w[32];
        tc::tmem_ld32(t_o + c, w);                          // the whole warp loads, valid rows store
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
