// Attention of few rows per sequence over a caller-owned paged cache (16-bit storage): decode steps, and chunks whose
// rows x query heads of a KV head fit one 16-row tensor-core tile.  (Two tiles, up to 32 rows, were slower than the tiled
// kernel of paged_chunk.cuh: 128 x 4 tokens on 1024 .. 6144, 28 on 4 heads of 128, 285 us against 207; 4 x 5 on 100 .. 300, 12 on
// 2 heads, 37 against 29.  With one tile it is the other way: 128 x 1 184 against 205, 4 x 1 22.5 against 29.)
//
// Bound by HBM: K and V of every visible page are read once per (sequence, KV head), all query heads of the group at
// once.  All pages of all (sequence, KV head) items form one list; every CTA takes an equal piece of it, whatever the
// lengths are, found on the device from the lengths alone.  A CTA's four warps walk the pages of their piece
// independently (warp w takes every fourth page; no barrier in the loop), each with its own ring of pages filled by
// 16-byte asynchronous copies; scores and P V run on mma.sync m16n8k16 with the online softmax in registers.  The
// warps' results are joined through shared memory at the end of an item; an item that runs over several CTAs leaves
// unnormalised parts, joined in piece order by split_merge_kernel.
//
// Measured (28 query on 4 KV heads of 128): one token for each of 128 sequences of 1024 .. 6144 tokens 164 to 171 us on different
// cards, 5.5 to 5.7 TB/s, 84 to 88 % of a copy's rate.  Beside 164: pages fetched as one bulk copy per row 212 us, as TMA boxes 168
// and 3.6 us of host time per tensor map; K and V of the new token written by a kernel of their own 3 us more.
//
// Weights are rounded to 16 bits before P V (sums of weights are not), as in the rollout's own attention and in the tiled
// kernel: against 64 bits the outputs are 1.9e-3 off, of which 1.65e-3 is their own rounding to 16 bits.  With a second 16-bit
// part of every weight the error is that 1.65e-3 alone, and the call above takes 179 us instead of 170.
#pragma once
#include "attn_tc.cuh"
#include "paged_kv.cuh"

namespace rpo {

// ---- items that are worked on in pieces ---------------------------------------------------------------------------
// CTA b's first and last pieces may belong to items that others work on too: slots 2 b and 2 b + 1.  An item's pieces
// lie in slot 2 b + 1 of the CTA b it begins in and in slot 2 c of every following CTA c.  CTA b records the item that
// begins in it and goes on behind it (n_parts 0: there is none).
struct SplitRec { int row0, head0, rows, n_parts; };       // rows: packed (token, head of the group), token-major

struct SplitWs {
  float* o;            // [slot][rows_cap][head_dim], unnormalised
  float2* ml;          // [slot][rows_cap]: running maximum (log2 domain) and sum
  SplitRec* rec;       // [CTA]
  int rows_cap;
};

template <typename T>
struct AttnOut { T* out; float* lse; int hq, rep; };

constexpr float LN2_F = 0.69314718055994531f, LOG2E_F = 1.44269504088896341f;

// o = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p over an item's pieces, added up in piece order.  Few pieces: a warp
// takes MERGE_ROWS rows at once, all of their loads in flight together.  Many (one long sequence): the warps of the CTA share a row's pieces, eight loads
// in flight each.
constexpr int MERGE_WARPS = 8, MERGE_LOADS = 8, MERGE_ROWS = 2, MERGE_FEW = 4;

template <typename T, int N>
__device__ __forceinline__ void merge_store(T* dst, const float (&x)[N], float scale) {
  T y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = from_f32<T>(x[i] * scale);
  if (sizeof(y) == 16) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(y);
  else if (sizeof(y) == 8) *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(y);
  else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(y);
}

template <typename T, int DH>
__global__ void __launch_bounds__(MERGE_WARPS * 32) split_merge_kernel(SplitWs ws, AttnOut<T> a) {
  constexpr int DPL = DH / 32, W = MERGE_WARPS;
  __shared__ float s_o[W][DH];
  __shared__ float s_l[W];
  const SplitRec rec = ws.rec[blockIdx.x];
  if (rec.n_parts == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, b = blockIdx.x;
  auto slot = [&](int p, int r) -> int64_t { return (int64_t)(p == 0 ? 2 * b + 1 : 2 * (b + p)) * ws.rows_cap + r; };
  auto load = [&](int64_t at, float (&x)[DPL]) {
#pragma unroll
    for (int i = 0; i < DPL; i += 2) { const float2 y = *reinterpret_cast<const float2*>(ws.o + at * DH + lane * DPL + i); x[i] = y.x; x[i + 1] = y.y; }
  };
  auto place = [&](int r) -> int64_t { return (int64_t)(rec.row0 + r / a.rep) * a.hq + rec.head0 + r % a.rep; };
  if (rec.n_parts <= MERGE_FEW) {
    for (int r0 = (blockIdx.y * W + warp) * MERGE_ROWS; r0 < rec.rows; r0 += gridDim.y * W * MERGE_ROWS) {
      float2 ml[MERGE_ROWS][MERGE_FEW];
      float x[MERGE_ROWS][MERGE_FEW][DPL];
#pragma unroll
      for (int p = 0; p < MERGE_FEW; ++p)
#pragma unroll
        for (int u = 0; u < MERGE_ROWS; ++u) {
          ml[u][p] = make_float2(-INFINITY, 0.f);
#pragma unroll
          for (int i = 0; i < DPL; ++i) x[u][p][i] = 0.f;
          if (p < rec.n_parts) {
            const int64_t at = slot(p, min(r0 + u, rec.rows - 1));
            ml[u][p] = ws.ml[at];
            load(at, x[u][p]);
          }
        }
#pragma unroll
      for (int u = 0; u < MERGE_ROWS; ++u) {
        if (r0 + u >= rec.rows) break;
        float m = -INFINITY, l = 0.f, acc[DPL];
#pragma unroll
        for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
#pragma unroll
        for (int p = 0; p < MERGE_FEW; ++p) m = fmaxf(m, ml[u][p].x);
        const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int p = 0; p < MERGE_FEW; ++p) {
          const float w = fa::ex2(ml[u][p].x - mu);
          l = fmaf(w, ml[u][p].y, l);
#pragma unroll
          for (int i = 0; i < DPL; ++i) acc[i] = fmaf(w, x[u][p][i], acc[i]);
        }
        const int64_t dst = place(r0 + u);
        merge_store(a.out + dst * DH + lane * DPL, acc, l > 0.f ? 1.0f / l : 0.f);
        if (lane == 0 && a.lse) a.lse[dst] = l > 0.f ? m * LN2_F + logf(l) : -INFINITY;
      }
    }
    return;
  }
  for (int r = blockIdx.y; r < rec.rows; r += gridDim.y) {
    float m = -INFINITY;
    for (int p = lane; p < rec.n_parts; p += 32) m = fmaxf(m, ws.ml[slot(p, r)].x);
    m = warp_max(m);
    const float mu = m == -INFINITY ? 0.f : m;
    float l = 0.f, acc[DPL];
#pragma unroll
    for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
    for (int p0 = warp; p0 < rec.n_parts; p0 += MERGE_LOADS * W) {
      float x[MERGE_LOADS][DPL];
      float2 ml[MERGE_LOADS];
#pragma unroll
      for (int u = 0; u < MERGE_LOADS; ++u) {
        const bool v = p0 + u * W < rec.n_parts;
        const int64_t at = slot(v ? p0 + u * W : p0, r);
        ml[u] = v ? ws.ml[at] : make_float2(-INFINITY, 0.f);
        load(at, x[u]);
      }
#pragma unroll
      for (int u = 0; u < MERGE_LOADS; ++u) {
        const float w = fa::ex2(ml[u].x - mu);
        l = fmaf(w, ml[u].y, l);
#pragma unroll
        for (int i = 0; i < DPL; ++i) acc[i] = fmaf(w, x[u][i], acc[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < DPL; ++i) s_o[warp][lane * DPL + i] = acc[i];
    if (lane == 0) s_l[warp] = l;
    __syncthreads();
    const int64_t dst = place(r);
    l = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) l += s_l[w];
    if ((int)threadIdx.x < DH) {
      float o = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) o += s_o[w][threadIdx.x];
      a.out[dst * DH + threadIdx.x] = from_f32<T>(l > 0.f ? o / l : 0.f);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[dst] = l > 0.f ? m * LN2_F + logf(l) : -INFINITY;
    __syncthreads();
  }
}

// ---- the keys a run of rows can see -------------------------------------------------------------------------------
// Positions [p0, p1] (p0 may be negative: rows before the first token).  Pages [0, n_first) hold the sinks (all pages
// when there is no window or it reaches them), pages [lo_page, end_page) the window; keys below `lo` that are no sinks
// are seen by none of the rows.
struct KeyPages {
  int n_first, lo_page, end_page, lo;
  __device__ __forceinline__ int count() const { return n_first + end_page - lo_page; }
  __device__ __forceinline__ int page(int i) const { return i < n_first ? i : lo_page + i - n_first; }
};

__device__ __forceinline__ KeyPages key_pages(const ChunkArgs& c, int p0, int p1) {
  KeyPages k;
  const int n = max(p1 + 1, 0);
  k.end_page = (n + KV_BLOCK - 1) / KV_BLOCK;
  k.lo = c.window > 0 ? max(0, p0 - c.window + 1) : 0;
  const int sinks = min(c.sinks, n);
  k.n_first = (sinks + KV_BLOCK - 1) / KV_BLOCK;
  k.lo_page = k.lo / KV_BLOCK;
  if (c.window <= 0 || k.lo_page <= k.n_first) { k.n_first = 0; k.lo_page = 0; if (k.lo <= sinks || c.window <= 0) k.lo = 0; }
  return k;
}

// The list of all pages: pref[s] = sum of count() over the sequences before s; returns the sum over all.  Called by all
// THREADS threads of the CTA (thread t: consecutive sequences); ends with a barrier.
template <int THREADS, typename F>
__device__ __forceinline__ int page_list(int n_seqs, int* pref, int* scan, F count) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per = (n_seqs + THREADS - 1) / THREADS;
  int sum = 0;
  for (int s = tid * per; s < min(n_seqs, (tid + 1) * per); ++s) { const int n = count(s); pref[s] = n; sum += n; }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int n = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += n; }
  if (lane == 31) scan[warp] = incl;
  __syncthreads();
  int run = incl - sum, total = 0;
  for (int w = 0; w < THREADS / 32; ++w) { if (w < warp) run += scan[w]; total += scan[w]; }
  for (int s = tid * per; s < min(n_seqs, (tid + 1) * per); ++s) { const int n = pref[s]; pref[s] = run; run += n; }
  __syncthreads();
  return total;
}
// The sequence whose pages hold place f of the list (empty sequences hold none).
__device__ __forceinline__ int page_list_seq(const int* pref, int n_seqs, int f) {
  int lo = 0, hi = n_seqs - 1;
  while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (pref[mid] <= f) lo = mid; else hi = mid - 1; }
  return lo;
}

template <int DH>
struct StepCfg {
  static constexpr int WARPS = 4;
  static constexpr int PAGE_BYTES = KV_BLOCK * DH * 2;                 // of K or of V
  static constexpr int STAGES = 3;
  static constexpr int RING = WARPS * STAGES * 2 * PAGE_BYTES;
  static constexpr int ROWS = 16;
  static constexpr int XO = DH + 4;                                    // floats per row of a warp's result in shared memory
  static constexpr int XCH = WARPS * ROWS * (XO + 2) * 4;
  static constexpr int SMEM = (RING > XCH ? RING : XCH);               // + (n_seqs + 1) ints
};

struct StepArgs {
  PagedView<bf16> kv; ChunkArgs c;
  const bf16* q; int64_t q_stride; float scale_log2;
  const bf16 *k_new, *v_new; int64_t new_stride;             // NULL: the chunk's K and V are in the cache
  AttnOut<bf16> o; SplitWs ws;
  int min_share;
};

template <int DH>
__global__ void __launch_bounds__(128, 2) paged_step_kernel(StepArgs a) {
  using Cfg = StepCfg<DH>;
  constexpr int ROWS = Cfg::ROWS, STAGES = Cfg::STAGES, PB = Cfg::PAGE_BYTES, KS = DH / 16, NT = DH / 8, CPR = DH / 8;
  extern __shared__ __align__(128) uint8_t st_smem[];
  int* s_pref = reinterpret_cast<int*>(st_smem + Cfg::SMEM);          // pages of all items of the sequences before s
  __shared__ int s_scan[4];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, tq = lane & 3;
  const int n_seqs = a.kv.n_seqs, hkv = a.kv.hkv, rep = a.o.rep;

  const int total = page_list<128>(n_seqs, s_pref, s_scan, [&](int s) {
    const ChunkSpan sp = chunk_span(a.kv, a.c, s);
    return sp.rows > 0 ? max(1, key_pages(a.c, sp.len - sp.rows, sp.len - 1).count()) * hkv : 0;
  });
  const int share = max(a.min_share, (total + (int)gridDim.x - 1) / (int)gridDim.x);
  const int f_end = (int)min((int64_t)total, (int64_t)(blockIdx.x + 1) * share);
  int f = (int)min((int64_t)total, (int64_t)blockIdx.x * share);
  if (tid == 0) a.ws.rec[blockIdx.x] = SplitRec{0, 0, 0, 0};

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(st_smem) + warp * (STAGES * 2 * PB);
  float* x_o = reinterpret_cast<float*>(st_smem);                      // results of the warps (the ring is idle then)
  float2* x_ml = reinterpret_cast<float2*>(st_smem + Cfg::WARPS * ROWS * Cfg::XO * 4);
  auto sw = [](int row, int chunk) -> uint32_t { return (uint32_t)(row * (DH * 2) + ((chunk ^ (row & 7)) << 4)); };

  while (f < f_end) {
    const int s = page_list_seq(s_pref, n_seqs, f);
    const ChunkSpan sp = chunk_span(a.kv, a.c, s);
    const int R = sp.rows * rep, p0 = sp.len - sp.rows, p1 = sp.len - 1;
    const KeyPages kp = key_pages(a.c, p0, p1);
    const int n_pages = max(1, kp.count()), in_seq = f - s_pref[s], h = in_seq / n_pages, i0 = in_seq % n_pages;
    const int i1 = min(n_pages, i0 + (f_end - f)), item0 = f - i0;     // my pages of the item, its place in the list
    bf16* kb = a.kv.k + h * a.kv.head_stride;
    bf16* vb = a.kv.v + h * a.kv.head_stride;
    const int32_t* tbl = a.kv.table + (int64_t)s * a.kv.table_stride;

    // ---- queries as A fragments: rows g, g + 8 of every 16
    uint32_t qf[KS][4];
    int prow[2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int r = hh * 8 + g;
      const bool v = r < R;
      prow[hh] = v ? p0 + r / rep : p1;
      const uint32_t* qp = reinterpret_cast<const uint32_t*>(a.q + (int64_t)(sp.row0 + (v ? r / rep : 0)) * a.q_stride + (h * rep + (v ? r % rep : 0)) * DH) + tq;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        qf[k][hh] = v ? qp[k * 8] : 0u;
        qf[k][hh + 2] = v ? qp[k * 8 + 4] : 0u;
      }
    }

    float o[NT][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NT; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    const int n_mine = (i1 - i0 - warp + 3) / 4;                       // pages i0 + warp, i0 + warp + 4, ...
    int ids = 0;                                                       // lane t: block of my page 32 b + t
    auto fetch_ids = [&](int base) {
      const int i = i0 + warp + 4 * (base + lane);
      ids = -1;
      if (i < i1 && kp.page(i) < kp.end_page) {
        ids = tbl[kp.page(i)];
        if (ids < 0 || ids >= a.kv.n_blocks) { atomicOr(a.kv.status, STATUS_BAD_BLOCK); ids = -1; }
      }
    };
    auto load = [&](int it) {                                          // page `it` of mine into stage it % STAGES
      const int blk = __shfl_sync(0xffffffffu, ids, it & 31);
      const int key0 = kp.page(i0 + warp + 4 * it) * KV_BLOCK;
      const uint32_t dst = ring + (it % STAGES) * (2 * PB);
      auto piece = [&](int e, bool fresh) {
        const int x = e * 32 + lane, row = x / CPR, ch = x % CPR, j = key0 + row;
        // rows that none of the queries sees become zeros: whatever the cache holds there, 0 x NaN included
        const int bytes = (blk >= 0 && j <= p1 && (j >= kp.lo || j < a.c.sinks)) ? 16 : 0;
        const int64_t at = ((int64_t)max(blk, 0) * KV_BLOCK + row) * DH + ch * 8;
        const bf16 *ks = kb + at, *vs = vb + at;
        if (fresh && j >= p0 && bytes) {
          // a row of the chunk: read where it is, and written to its page on the way (this page is nobody else's)
          const int64_t n = (int64_t)(sp.row0 + j - p0) * a.new_stride + h * DH + ch * 8;
          ks = a.k_new + n; vs = a.v_new + n;
          *reinterpret_cast<uint4*>(kb + at) = *reinterpret_cast<const uint4*>(ks);
          *reinterpret_cast<uint4*>(vb + at) = *reinterpret_cast<const uint4*>(vs);
        }
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + sw(row, ch)), "l"(ks), "r"(bytes) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + PB + sw(row, ch)), "l"(vs), "r"(bytes) : "memory");
      };
      if (a.k_new && key0 + KV_BLOCK > p0) {
#pragma unroll 1
        for (int e = 0; e < KV_BLOCK * CPR / 32; ++e) piece(e, true);
      } else {
#pragma unroll
        for (int e = 0; e < KV_BLOCK * CPR / 32; ++e) piece(e, false);
      }
    };
    if (n_mine > 0) fetch_ids(0);
#pragma unroll
    for (int it = 0; it < STAGES - 1; ++it) { if (it < n_mine) load(it); fa::cp_commit(); }
    for (int it = 0; it < n_mine; ++it) {
      if (it + STAGES - 1 < n_mine) {
        if (((it + STAGES - 1) & 31) == 0) fetch_ids(it + STAGES - 1);
        load(it + STAGES - 1);
      }
      fa::cp_commit();
      fa::cp_wait<STAGES - 1>();
      __syncwarp();
      const uint32_t sk = ring + (it % STAGES) * (2 * PB), sv = sk + PB;
      float sc[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t b0, b1, b2, b3;
        fa::ldsm_x4(sk + sw(((lane >> 4) << 3) + (lane & 7), k * 2 + ((lane >> 3) & 1)), b0, b1, b2, b3);
        fa::mma_bf16(sc[0], qf[k], b0, b1);
        fa::mma_bf16(sc[1], qf[k], b2, b3);
      }
      const int key0 = kp.page(i0 + warp + 4 * it) * KV_BLOCK;
      const bool whole = key0 + KV_BLOCK - 1 <= p0 && (a.c.window <= 0 || key0 > p1 - a.c.window || key0 + KV_BLOCK <= a.c.sinks);
      uint32_t pf[4];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        float x[4] = {sc[0][2 * hh], sc[0][2 * hh + 1], sc[1][2 * hh], sc[1][2 * hh + 1]};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] *= a.scale_log2;
          if (!whole && !chunk_visible(a.c, key0 + (e >> 1) * 8 + tq * 2 + (e & 1), prow[hh])) x[e] = -INFINITY;
        }
        float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        // the reference maximum moves when it is outgrown; the sums are exact for any reference
        const float mn = fmaxf(m[hh], mx);
        if (__any_sync(0xffffffffu, mn > m[hh])) {
          const float corr = mn == -INFINITY ? 1.f : fa::ex2(m[hh] - mn);
          l[hh] *= corr;
          m[hh] = mn;
#pragma unroll
          for (int n = 0; n < NT; ++n) { o[n][2 * hh] *= corr; o[n][2 * hh + 1] *= corr; }
        }
        const float mu = m[hh] == -INFINITY ? 0.f : m[hh];
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = fa::ex2(x[e] - mu); l[hh] += x[e]; }
        pf[hh] = fa::pack_bf16(x[0], x[1]);
        pf[hh + 2] = fa::pack_bf16(x[2], x[3]);
      }
#pragma unroll
      for (int n = 0; n < NT; n += 2) {
        uint32_t b0, b1, b2, b3;
        fa::ldsm_x4_t(sv + sw((((lane >> 3) & 1) << 3) + (lane & 7), n + (lane >> 4)), b0, b1, b2, b3);
        fa::mma_bf16(o[n], pf, b0, b1);
        fa::mma_bf16(o[n + 1], pf, b2, b3);
      }
      __syncwarp();
    }
    fa::cp_wait<0>();
    __syncthreads();

    // ---- join the warps
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int r = hh * 8 + g;
      float ls = l[hh];
      ls += __shfl_xor_sync(0xffffffffu, ls, 1);
      ls += __shfl_xor_sync(0xffffffffu, ls, 2);
      if (tq == 0) x_ml[warp * ROWS + r] = make_float2(m[hh], ls);
      if (r < R)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          *reinterpret_cast<float2*>(x_o + (warp * ROWS + r) * Cfg::XO + n * 8 + tq * 2) = make_float2(o[n][2 * hh], o[n][2 * hh + 1]);
    }
    __syncthreads();
    const bool begins = i0 == 0, ends = i1 == n_pages;
    const int slot = begins ? 2 * blockIdx.x + 1 : 2 * blockIdx.x;
    for (int x = tid; x < R * (DH / 2); x += 128) {
      const int r = x / (DH / 2), d = (x % (DH / 2)) * 2;
      float2 ml[4];
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) { ml[w] = x_ml[w * ROWS + r]; mm = fmaxf(mm, ml[w].x); }
      const float mu = mm == -INFINITY ? 0.f : mm;
      float ls = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float wt = fa::ex2(ml[w].x - mu);
        const float2 v = *reinterpret_cast<const float2*>(x_o + (w * ROWS + r) * Cfg::XO + d);
        ls = fmaf(wt, ml[w].y, ls); y0 = fmaf(wt, v.x, y0); y1 = fmaf(wt, v.y, y1);
      }
      if (begins && ends) {
        const int64_t dst = (int64_t)(sp.row0 + r / rep) * a.o.hq + h * rep + r % rep;
        const float inv = ls > 0.f ? 1.0f / ls : 0.f;
        *reinterpret_cast<uint32_t*>(a.o.out + dst * DH + d) = fa::pack_bf16(y0 * inv, y1 * inv);
        if (d == 0 && a.o.lse) a.o.lse[dst] = ls > 0.f ? mm * LN2_F + logf(ls) : -INFINITY;
      } else {
        const int64_t at = (int64_t)slot * a.ws.rows_cap + r;
        *reinterpret_cast<float2*>(a.ws.o + at * DH + d) = make_float2(y0, y1);
        if (d == 0) a.ws.ml[at] = make_float2(mm, ls);
      }
    }
    if (begins && !ends && tid == 0)
      a.ws.rec[blockIdx.x] = SplitRec{sp.row0, h * rep, R, (item0 + n_pages - 1) / share - (int)blockIdx.x + 1};
    __syncthreads();
    f += i1 - i0;
  }
}

}  // namespace rpo
