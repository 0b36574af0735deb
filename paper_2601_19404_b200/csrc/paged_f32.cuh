// The operators on a caller-owned paged cache for 32-bit storage, on CUDA cores: products stay exact to float32, which
// the tensor cores' 16-bit or tf32 inputs would not give.
//
// Same items, pieces and merge as the 16-bit kernels (paged_chunk.cuh).  256 threads as 16 x 16: thread (ty, tx) owns
// TM = BM / 16 consecutive rows and the keys tx, tx + 16, ... of a tile, then the same rows and 4 (or 2 x 4) output dims.
// Operands are read from shared memory as float4: per four dims 4 TM multiply-adds for each of its keys against TM + KPT
// loads.  A float4 load takes four passes of shared memory whatever it shares, so the loads bound both variants: with BM = 64
// (64 multiply-adds per 4 + 4 loads) they take twice the time of the multiply-adds, with BM = 16, which serves decode steps,
// more.  K and V of the next tile are fetched (cp.async, zero-filled where no row looks) while the other half of this tile
// is worked on.  Measured: 3 chunks of up to 777 tokens behind up to 1500, window 500, 4 on 2 heads of 64: 64 us (18 % of the
// nominal multiply-add rate), their attention mass 113; one token for each of 32 sequences of 1024 .. 4096, 12 on 2 heads of 128: 154 us
// (19 % of a copy's rate), their mass 80.
#pragma once
#include "paged_chunk.cuh"

namespace rpo {

struct F32Args {
  PagedView<float> kv; ChunkArgs c;
  const float* q; int64_t q_stride; float scale_log2;
  AttnOut<float> o; SplitWs ws;
  const ChunkItem* items; const ChunkPlan* plan;
  int tok;                                                   // tokens per item
};

template <int DH, int BM>
struct F32Cfg {
  static constexpr int BN = DH == 64 ? 64 : 32;              // keys per tile: two or three CTAs fit an SM
  static constexpr int QS = DH + 4, PS = BN + 4;             // padded rows: the 8 rows a quarter-warp reads hit all banks
  static constexpr int SMEM = (BM * QS + BN * QS + BN * DH + BM * PS) * 4;
  static constexpr int CTAS = DH == 64 ? 3 : 2;
};

__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}

// Scores of TM rows against KPT keys: acc[i][j] = q_(r0 + i) . k_(tx + 16 j).
template <int DH, int TM, int KPT>
__device__ __forceinline__ void f32_scores(const float* sq, const float* sk, int r0, int tx, float (&acc)[TM][KPT]) {
  constexpr int S = DH + 4;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < KPT; ++j) acc[i][j] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DH; d += 4) {
    float4 q[TM], k[KPT];
#pragma unroll
    for (int i = 0; i < TM; ++i) q[i] = *reinterpret_cast<const float4*>(sq + (r0 + i) * S + d);
#pragma unroll
    for (int j = 0; j < KPT; ++j) k[j] = *reinterpret_cast<const float4*>(sk + (tx + 16 * j) * S + d);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < KPT; ++j) {
        acc[i][j] = fmaf(q[i].x, k[j].x, acc[i][j]);
        acc[i][j] = fmaf(q[i].y, k[j].y, acc[i][j]);
        acc[i][j] = fmaf(q[i].z, k[j].z, acc[i][j]);
        acc[i][j] = fmaf(q[i].w, k[j].w, acc[i][j]);
      }
  }
}

// TREE: the chunks are trees (paged_tree.cuh).
template <int DH, int BM, bool TREE>
__global__ void __launch_bounds__(256, F32Cfg<DH, BM>::CTAS) paged_f32_kernel(F32Args a) {
  using Cfg = F32Cfg<DH, BM>;
  constexpr int NO_NODE = -(1 << 30);                      // below every position (those of a tree longer than its sequence may be negative)
  constexpr int BN = Cfg::BN, TM = BM / 16, KPT = BN / 16, DG = DH / 64, QS = Cfg::QS, PS = Cfg::PS, CPR = DH / 4, LD = BN * CPR / 256;
  extern __shared__ __align__(16) float f32_smem[];
  float *sq = f32_smem, *sk = sq + BM * QS, *sv = sk + BN * QS, *sp = sv + BN * DH;
  __shared__ int s_first;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, r0 = ty * TM, hkv = a.kv.hkv, rep = a.o.rep;
  const ChunkPlan plan = *a.plan;
  if (tid == 0) { a.ws.rec[blockIdx.x] = SplitRec{0, 0, 0, 0}; s_first = 0; }
  PieceWalk walk;
  walk.items = a.items; walk.hkv = hkv; walk.over = plan.over;
  walk.f = (int)min((int64_t)plan.total, (int64_t)blockIdx.x * plan.share);
  walk.f_end = (int)min((int64_t)plan.total, (int64_t)(blockIdx.x + 1) * plan.share);
  __syncthreads();
  if (walk.f < walk.f_end)
    for (int i = tid; i < plan.n_items; i += 256) {
      const int2 x = *reinterpret_cast<const int2*>(a.items + i);
      if (x.x <= walk.f && walk.f < x.x + (x.y + plan.over) * hkv) s_first = i;
    }
  __syncthreads();
  walk.idx = s_first;
  const uint32_t uq = (uint32_t)__cvta_generic_to_shared(sq), uk = (uint32_t)__cvta_generic_to_shared(sk), uv = (uint32_t)__cvta_generic_to_shared(sv);

  while (walk.next()) {
    const int R = walk.it.n_tok * rep, p0 = walk.it.p0, p1 = p0 + walk.it.n_tok - 1;
    const KeyTiles<BN / KV_BLOCK> kt(a.c, walk.it.key0, p1);
    const TreeRow* nodes = TREE ? a.c.tree + (walk.it.row0 - (p0 - walk.it.key0)) : nullptr;      // the sequence's first node
    const int32_t* tbl = a.kv.table + (int64_t)walk.it.seq * a.kv.table_stride;
    const float* kb = a.kv.k + walk.head * a.kv.head_stride;
    const float* vb = a.kv.v + walk.head * a.kv.head_stride;
    int blk[BN / KV_BLOCK], blk_next[BN / KV_BLOCK];
    auto lookup = [&](int t, int (&b)[BN / KV_BLOCK]) {
#pragma unroll
      for (int i = 0; i < BN / KV_BLOCK; ++i) {
        const int page = kt.page0(t) + i;
        b[i] = -1;
        if (page < kt.page_end(t)) {
          b[i] = tbl[page];
          if (b[i] < 0 || b[i] >= a.kv.n_blocks) { if (tid == 0) atomicOr(a.kv.status, STATUS_BAD_BLOCK); b[i] = -1; }
        }
      }
    };
    auto load = [&](uint32_t dst, int stride, const float* base, int t, const int (&b)[BN / KV_BLOCK]) {
      const int key0 = kt.page0(t) * KV_BLOCK, end = t < kt.n1 ? min(a.c.sinks, p1 + 1) : p1 + 1;
#pragma unroll
      for (int e = 0; e < LD; ++e) {
        const int x = e * 256 + tid, row = x / CPR, ch = x % CPR, j = key0 + row, bk = b[e * 256 / CPR / KV_BLOCK];
        const bool live = bk >= 0 && j < end && (j >= kt.kp.lo || j < a.c.sinks) && !(TREE && j >= walk.it.key0 && nodes[j - walk.it.key0].depth < 0);
        cp_async16_zfill(dst + (row * stride + ch * 4) * 4, base + ((int64_t)max(bk, 0) * KV_BLOCK + row % KV_BLOCK) * DH + ch * 4, live);
      }
      fa::cp_commit();
    };
    for (int x = tid; x < BM * CPR; x += 256) {
      const int r = x / CPR, ch = x % CPR;
      const bool live = r < R;
      cp_async16_zfill(uq + (r * QS + ch * 4) * 4, a.q + (int64_t)(walk.it.row0 + (live ? r / rep : 0)) * a.q_stride + (walk.head * rep + (live ? r % rep : 0)) * DH + ch * 4, live);
    }
    lookup(walk.t0, blk);
    load(uk, QS, kb, walk.t0, blk);                          // (one group with the queries)
    load(uv, DH, vb, walk.t0, blk);
    float o[TM][DG][4], m[TM], l[TM];
    int prow[TM];
    const TreeRow* node[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      m[i] = -INFINITY; l[i] = 0.f;
      prow[i] = min(p0 + (r0 + i) / rep, p1);
      if (TREE) {
        node[i] = nodes + (prow[i] - walk.it.key0);
        prow[i] = node[i]->depth < 0 ? NO_NODE : walk.it.key0 + node[i]->depth;
      }
#pragma unroll
      for (int g = 0; g < DG; ++g) o[i][g][0] = o[i][g][1] = o[i][g][2] = o[i][g][3] = 0.f;
    }
    for (int t = walk.t0; t < walk.t1; ++t) {
      if (t + 1 < walk.t1) lookup(t + 1, blk_next);
      fa::cp_wait<1>();                                      // K of this tile (V may be on its way)
      __syncthreads();
      float s[TM][KPT];
      f32_scores<DH, TM, KPT>(sq, sk, r0, tx, s);
      __syncthreads();                                       // K is read: the next one may come
      if (t + 1 < walk.t1) load(uk, QS, kb, t + 1, blk_next); else fa::cp_commit();
      const int key0 = kt.page0(t) * KV_BLOCK;
      const bool first_range = t < kt.n1;
      const int p_whole = TREE ? walk.it.key0 - 1 : p0;
      const bool whole = key0 + BN - 1 <= (first_range ? min(p_whole, a.c.sinks - 1) : p_whole) &&
                         (a.c.window <= 0 || key0 > p1 - a.c.window || key0 + BN <= a.c.sinks);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
          s[i][j] *= a.scale_log2;
          const int key = key0 + tx + 16 * j;
          if (TREE && !whole && key >= walk.it.key0) {
            const int slot = key - walk.it.key0;
            if (prow[i] == NO_NODE || first_range || slot >= TREE_MAX_NODES || !((node[i]->seen[slot >> 5] >> (slot & 31)) & 1)) s[i][j] = -INFINITY;
          } else if (!whole && (!chunk_visible(a.c, key, prow[i]) || (first_range && key >= a.c.sinks))) s[i][j] = -INFINITY;
          mx = fmaxf(mx, s[i][j]);
        }
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
        const float mn = fmaxf(m[i], mx), mu = mn == -INFINITY ? 0.f : mn;
        const float corr = fa::ex2(m[i] - mu);
        m[i] = mn;
        l[i] *= corr;
#pragma unroll
        for (int g = 0; g < DG; ++g)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[i][g][x] *= corr;
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
          const float p = fa::ex2(s[i][j] - mu);
          l[i] += p;
          sp[(r0 + i) * PS + tx + 16 * j] = p;
        }
      }
      fa::cp_wait<1>();                                      // V of this tile
      __syncthreads();
#pragma unroll 4
      for (int k = 0; k < BN; k += 4) {
        float4 p[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) p[i] = *reinterpret_cast<const float4*>(sp + (r0 + i) * PS + k);
#pragma unroll
        for (int g = 0; g < DG; ++g)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const float4 v = *reinterpret_cast<const float4*>(sv + (k + kk) * DH + g * 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
              const float w = kk == 0 ? p[i].x : kk == 1 ? p[i].y : kk == 2 ? p[i].z : p[i].w;
              o[i][g][0] = fmaf(w, v.x, o[i][g][0]); o[i][g][1] = fmaf(w, v.y, o[i][g][1]);
              o[i][g][2] = fmaf(w, v.z, o[i][g][2]); o[i][g][3] = fmaf(w, v.w, o[i][g][3]);
            }
          }
      }
      __syncthreads();                                       // V is read
      if (t + 1 < walk.t1) load(uv, DH, vb, t + 1, blk_next); else fa::cp_commit();
    }
    fa::cp_wait<0>();
    const bool begins = walk.t0 == 0, ends = walk.t1 == walk.it.n_tiles, split = !(begins && ends);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
      const int r = r0 + i;
      if (r >= R) continue;
      if (TREE && prow[i] == NO_NODE) {                       // no node: whatever the tiles without masks gave
        m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
        for (int g = 0; g < DG; ++g) o[i][g][0] = o[i][g][1] = o[i][g][2] = o[i][g][3] = 0.f;
      }
      const int64_t dst = (int64_t)(walk.it.row0 + r / rep) * a.o.hq + walk.head * rep + r % rep;
      const int64_t part = (int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * a.ws.rows_cap + r;
      const float inv = split ? 1.f : l[i] > 0.f ? 1.0f / l[i] : 0.f;
      float* to = split ? a.ws.o + part * DH : a.o.out + dst * DH;
#pragma unroll
      for (int g = 0; g < DG; ++g)
        *reinterpret_cast<float4*>(to + g * 64 + tx * 4) = make_float4(o[i][g][0] * inv, o[i][g][1] * inv, o[i][g][2] * inv, o[i][g][3] * inv);
      if (tx == 0) {
        if (split) a.ws.ml[part] = make_float2(m[i], l[i]);
        else if (a.o.lse) a.o.lse[dst] = l[i] > 0.f ? m[i] * LN2_F + logf(l[i]) : -INFINITY;
      }
    }
    if (begins && !ends && tid == 0)
      a.ws.rec[blockIdx.x] = SplitRec{walk.it.row0, walk.head * rep, R, walk.parts(plan.share, blockIdx.x)};
    __syncthreads();                                         // the next piece overwrites Q, K and V
  }
}

// Attention mass, 32-bit: a CTA takes 64 keys of one (sequence, KV head) at a time and walks the rows that see any of them.  Thread
// (ty, tx) sums its rows' weights for its keys; the sixteen ty of a key are added up in order at the end.
struct MassF32Args {
  PagedView<float> kv; ChunkArgs c;
  const float* q; int64_t q_stride; float scale_log2;
  const float* lse; const float* in; float* out; int stride, rep;
};

constexpr int MF_KEYS = 64;

template <int DH, int BM>
__global__ void __launch_bounds__(256) mass_f32_kernel(MassF32Args a) {
  constexpr int TM = BM / 16, KPT = MF_KEYS / 16, S = DH + 4, CPR = DH / 4;
  extern __shared__ __align__(16) float mf_smem[];
  float *sk = mf_smem, *sq = sk + MF_KEYS * S, *s_lse = sq + 2 * BM * S;      // two buffers of rows and log-sums
  const int s = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, rep = a.rep;
  const ChunkSpan sp = chunk_span(a.kv, a.c, s);
  const int live = min(sp.len, a.stride);
  if (sp.len > a.stride && tid == 0) atomicOr(a.kv.status, STATUS_BAD_LENGTH);
  const int p0 = sp.len - sp.rows, p1 = sp.len - 1;
  const KeyPages kp = key_pages(a.c, p0, p1);
  const int32_t* tbl = a.kv.table + (int64_t)s * a.kv.table_stride;
  const uint32_t uk = (uint32_t)__cvta_generic_to_shared(sk), uq = (uint32_t)__cvta_generic_to_shared(sq), ul = (uint32_t)__cvta_generic_to_shared(s_lse);
  for (int key0 = blockIdx.x * MF_KEYS; key0 < live; key0 += gridDim.x * MF_KEYS) {
    // tokens that see any of the keys
    const int tok0 = max(0, key0 - p0);
    int tok1 = sp.rows;
    if (a.c.window > 0 && key0 >= a.c.sinks) tok1 = (int)min((int64_t)tok1, max((int64_t)0, (int64_t)key0 + MF_KEYS - 1 + a.c.window - p0));
    const int r_end = tok1 * rep;
    auto load_rows = [&](int base, int buf) {                  // BM rows and their log-sums
#pragma unroll
      for (int e = 0; e < BM * CPR / 256; ++e) {
        const int x = e * 256 + tid, r = base + x / CPR, ch = x % CPR;
        const bool there = r < r_end;
        cp_async16_zfill(uq + (buf * BM * S + (x / CPR) * S + ch * 4) * 4,
                         a.q + (int64_t)(sp.row0 + (there ? r / rep : 0)) * a.q_stride + (h * rep + (there ? r % rep : 0)) * DH + ch * 4, there);
      }
      if (tid < BM && base + tid < r_end) {
        const int r = base + tid;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(ul + (buf * BM + tid) * 4), "l"(a.lse + (int64_t)(sp.row0 + r / rep) * a.c.hq + h * rep + r % rep) : "memory");
      }
      fa::cp_commit();
    };
    __syncthreads();                                           // the last tile's keys and sums are read
    int blk[MF_KEYS / KV_BLOCK];
#pragma unroll
    for (int i = 0; i < MF_KEYS / KV_BLOCK; ++i) {
      const int page = key0 / KV_BLOCK + i;
      blk[i] = -1;
      if (sp.rows > 0 && (page < kp.n_first || (page >= kp.lo_page && page < kp.end_page))) {
        blk[i] = tbl[page];
        if (blk[i] < 0 || blk[i] >= a.kv.n_blocks) { if (tid == 0) atomicOr(a.kv.status, STATUS_BAD_BLOCK); blk[i] = -1; }
      }
    }
#pragma unroll
    for (int e = 0; e < MF_KEYS * CPR / 256; ++e) {
      const int x = e * 256 + tid, row = x / CPR, ch = x % CPR, bk = blk[e * 256 / CPR / KV_BLOCK];
      cp_async16_zfill(uk + (row * S + ch * 4) * 4, a.kv.k + h * a.kv.head_stride + ((int64_t)max(bk, 0) * KV_BLOCK + row % KV_BLOCK) * DH + ch * 4, bk >= 0);
    }
    fa::cp_commit();                                           // a group of their own: waited for even if no row follows
    float sum[KPT];
#pragma unroll
    for (int j = 0; j < KPT; ++j) sum[j] = 0.f;
    int buf = 0;
    if (tok0 * rep < r_end) load_rows(tok0 * rep, 0);
    for (int base = tok0 * rep; base < r_end; base += BM, buf ^= 1) {
      if (base + BM < r_end) load_rows(base + BM, buf ^ 1); else fa::cp_commit();
      fa::cp_wait<1>();
      __syncthreads();
      float acc[TM][KPT];
      f32_scores<DH, TM, KPT>(sq + buf * BM * S, sk, ty * TM, tx, acc);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int r = base + ty * TM + i, p = r < r_end ? p0 + r / rep : -1;
        const float ls = s_lse[buf * BM + ty * TM + i] * LOG2E_F;
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
          const float w = fa::ex2(fmaf(acc[i][j], a.scale_log2, -ls));
          sum[j] += chunk_visible(a.c, key0 + tx + 16 * j, p) ? w : 0.f;
        }
      }
      __syncthreads();                                         // the buffer may be filled again
    }
    fa::cp_wait<0>();
    __syncthreads();
    float* part = sq;                                          // [16][64]
#pragma unroll
    for (int j = 0; j < KPT; ++j) part[ty * MF_KEYS + tx + 16 * j] = sum[j];
    __syncthreads();
    if (tid < MF_KEYS && key0 + tid < live) {
      float x = 0.f;
#pragma unroll
      for (int y = 0; y < 16; ++y) x += part[y * MF_KEYS + tid];
      const int64_t at = ((int64_t)s * a.kv.hkv + h) * a.stride + key0 + tid;
      a.out[at] = (a.in ? a.in[at] : 0.f) + x;
    }
  }
}

}  // namespace rpo
