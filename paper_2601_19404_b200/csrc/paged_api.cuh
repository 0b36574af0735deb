// Entry points of the operators on a caller-owned paged cache (part of rpo_api.cu).
#pragma once

// These calls run between kernels of the caller, not between the library's own: launched plainly, without the
// programmatic attribute (their kernels do not wait for a predecessor).
#define LAUNCH_OP(ctx, kern, grid, block, smem, ...)                                       \
  do {                                                                                     \
    prof_begin(ctx, #kern);                                                                \
    kern<<<dim3(grid), dim3(block), (size_t)(smem), (ctx)->stream>>>(__VA_ARGS__);         \
    prof_end(ctx);                                                                         \
    (ctx)->launches++;                                                                     \
    CUDA_TRY(cudaGetLastError());                                                          \
  } while (0)

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

static int check_paged(const rpo_ctx* c, const rpo_paged_kv* kv) {
  if (!c || !kv || !kv->d_k || !kv->d_v || !kv->d_block_table || !kv->d_lens || kv->n_blocks <= 0 || kv->n_seqs <= 0 ||
      kv->table_stride <= 0 || kv->n_kv_heads <= 0 || !aligned16(kv->d_k) || !aligned16(kv->d_v))
    return RPO_ERR_INVALID_ARG;
  if (kv->head_dim != 64 && kv->head_dim != 128) return RPO_ERR_SHAPE;
  if ((int64_t)kv->n_kv_heads * kv->n_blocks >= ((int64_t)1 << 31) / KV_BLOCK || kv->table_stride >= (1 << 26)) return RPO_ERR_LIMIT;
  return RPO_OK;
}

constexpr int OP_MAX_REP = 64;

static int check_chunk(const rpo_ctx* c, const rpo_paged_kv* kv, int n_rows, int hq, int max_chunk, const void* d_q, int64_t q_stride,
                       const int32_t* d_q_offsets, const rpo_chunk_cfg* cfg) {
  RPO_TRY(check_paged(c, kv));
  if (n_rows < 0 || hq <= 0 || max_chunk <= 0 || (n_rows > 0 && !d_q) || !d_q_offsets || !cfg || !(cfg->scale > 0.f) || std::isinf(cfg->scale * 1.5f) ||
      cfg->window < 0 || cfg->sinks < 0 || !aligned16(d_q) || (q_stride * (int64_t)c->esz) % 16)
    return RPO_ERR_INVALID_ARG;
  if (hq % kv->n_kv_heads || hq / kv->n_kv_heads > OP_MAX_REP) return RPO_ERR_SHAPE;
  if (n_rows > 1 && q_stride < (int64_t)hq * kv->head_dim) return RPO_ERR_INVALID_ARG;
  if (kv->n_seqs > OP_MAX_SEQS || (int64_t)n_rows * hq >= ((int64_t)1 << 30) ||
      (int64_t)kv->n_seqs * kv->table_stride * kv->n_kv_heads >= ((int64_t)1 << 31) - (1 << 20))
    return RPO_ERR_LIMIT;
  return RPO_OK;
}

template <typename T>
static PagedView<T> paged_view(rpo_ctx* c, const rpo_paged_kv* kv) {
  PagedView<T> v;
  v.k = (T*)kv->d_k; v.v = (T*)kv->d_v; v.table = kv->d_block_table; v.lens = kv->d_lens;
  v.head_stride = (int64_t)kv->n_blocks * KV_BLOCK * kv->head_dim;
  v.n_blocks = kv->n_blocks; v.n_seqs = kv->n_seqs; v.table_stride = kv->table_stride; v.hkv = kv->n_kv_heads; v.status = c->d_status;
  return v;
}

static ChunkArgs chunk_args(int n_rows, int hq, int max_chunk, const int32_t* offsets, const rpo_chunk_cfg* cfg) {
  ChunkArgs a;
  // positions lie in (-2^30, 2^30): a longer window or more sinks see no more, and sums with them stay in 32 bits
  constexpr int32_t most = 1 << 30;
  a.offsets = offsets; a.n_rows = n_rows; a.max_chunk = max_chunk; a.window = std::min(cfg->window, most); a.sinks = std::min(cfg->sinks, most); a.hq = hq;
  return a;
}

static SplitWs split_ws(rpo_ctx* c, int rows_cap) {
  SplitWs w;
  w.o = c->ws.op_part_o; w.ml = (float2*)c->ws.op_part_ml; w.rec = (SplitRec*)c->ws.op_rec; w.rows_cap = rows_cap;
  return w;
}

// Few rows per sequence (decode steps): one CTA pair per SM over an equal share of all pages.
template <int DH>
static int chunk_steps(rpo_ctx* c, const PagedView<bf16>& view, const ChunkArgs& a, const bf16* q, int64_t q_stride, const bf16* k_new, const bf16* v_new,
                       int64_t new_stride, float scale, bf16* out, float* lse) {
  using Cfg = StepCfg<DH>;
  CUDA_TRY((allow_smem<paged_step_kernel<DH>>(c, Cfg::SMEM + (OP_MAX_SEQS + 1) * 4)));
  const int grid = 2 * c->sm_count;
  StepArgs s;
  s.kv = view; s.c = a; s.q = q; s.q_stride = q_stride; s.k_new = k_new; s.v_new = v_new; s.new_stride = new_stride; s.scale_log2 = scale * 1.4426950408889634f;
  s.o.out = out; s.o.lse = lse; s.o.hq = a.hq; s.o.rep = a.hq / view.hkv; s.ws = split_ws(c, Cfg::ROWS); s.min_share = 4;
  LAUNCH_OP(c, (paged_step_kernel<DH>), grid, 128, Cfg::SMEM + (view.n_seqs + 1) * 4, s);
  LAUNCH_OP(c, (split_merge_kernel<bf16, DH>), dim3(grid, std::min(a.max_chunk * s.o.rep, Cfg::ROWS)), MERGE_WARPS * 32, 0, s.ws, s.o);
  return RPO_OK;
}

// Tensor map over rows of head_dim 16-bit values in 128-byte swizzled boxes: 2 or 3 dimensions.
static int op_map(rpo_ctx* c, CUtensorMap* m, const void* ptr, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  TcState* s = (TcState*)c->tc_state;
  if (!s || !s->encode) return RPO_ERR_CUDA;
  const cuuint32_t ones[3] = {1, 1, 1};
  return s->encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(ptr), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? RPO_OK : RPO_ERR_CUDA;
}
// Pages of K or V: one box is 16 tokens x 64 dims.
static int op_map_pages(rpo_ctx* c, CUtensorMap* m, const PagedView<bf16>& v, const bf16* base, int dh) {
  const cuuint64_t dims[2] = {(cuuint64_t)dh, (cuuint64_t)v.hkv * v.n_blocks * KV_BLOCK}, strides[1] = {(cuuint64_t)dh * 2};
  const cuuint32_t box[2] = {64, KV_BLOCK};
  return op_map(c, m, base, 2, dims, strides, box);
}
// Queries: one box is `tok` tokens x the rep heads of a KV head x 64 dims.
static int op_map_rows(rpo_ctx* c, CUtensorMap* m, const bf16* q, int64_t q_stride, int n_rows, int hq, int dh, int rep, int tok) {
  const cuuint64_t dims[3] = {(cuuint64_t)dh, (cuuint64_t)hq, (cuuint64_t)n_rows};
  const cuuint64_t strides[2] = {(cuuint64_t)dh * 2, (cuuint64_t)(n_rows > 1 ? q_stride : (int64_t)hq * dh) * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)rep, (cuuint32_t)tok};
  return op_map(c, m, q, 3, dims, strides, box);
}

// One CTA for the list of items, up to two per SM for the chunk's K and V.
template <typename T, int DH>
static int prepare_grid(const PagedView<T>& view, const ChunkArgs& a, const T* k_new) {
  return 1 + (k_new ? grid_for((int64_t)a.n_rows * view.hkv * 2 * (DH * sizeof(T) / 16), 1024, 2 * 148) : 0);
}

// Many rows per sequence: tensor-core tiles of 2 x (tokens x heads of a KV head <= 128) rows against 128 keys.
template <int DH>
static int chunk_tiles(rpo_ctx* c, const PagedView<bf16>& view, const ChunkArgs& a, const bf16* q, int64_t q_stride, const bf16* k_new, const bf16* v_new,
                      int64_t new_stride, float scale, bf16* out, float* lse) {
  using Cfg = ChunkCfg<DH>;
  CUDA_TRY((allow_smem<paged_chunk_kernel<DH>>(c, Cfg::SMEM)));
  ChunkTcArgs t;
  t.kv = view; t.c = a; t.scale_log2 = scale * 1.4426950408889634f;
  t.o.out = out; t.o.lse = lse; t.o.hq = a.hq; t.o.rep = a.hq / view.hkv; t.ws = split_ws(c, OP_PART_ROWS);
  t.tq = CH_BM / t.o.rep;
  if ((int64_t)a.n_rows / (2 * t.tq) + view.n_seqs > OP_MAX_ITEMS) return RPO_ERR_LIMIT;
  ChunkItem* items = (ChunkItem*)c->ws.op_items;
  ChunkPlan* plan = (ChunkPlan*)(items + OP_MAX_ITEMS);
  t.items = items; t.plan = plan;
  CUtensorMap qm, km, vm;
  RPO_TRY(op_map_rows(c, &qm, q, q_stride, a.n_rows, a.hq, DH, t.o.rep, t.tq));
  RPO_TRY(op_map_pages(c, &km, view, view.k, DH));
  RPO_TRY(op_map_pages(c, &vm, view, view.v, DH));
  LAUNCH_OP(c, (chunk_prepare_kernel<bf16, DH, CH_BN / KV_BLOCK>), (prepare_grid<bf16, DH>(view, a, k_new)), 1024, view.n_seqs * 4, view, a, 2 * t.tq, c->sm_count, 4,
            2, items, plan, k_new, v_new, new_stride);
  LAUNCH_OP(c, (paged_chunk_kernel<DH>), c->sm_count, Cfg::THREADS, Cfg::SMEM, qm, km, vm, t);
  LAUNCH_OP(c, (split_merge_kernel<bf16, DH>), dim3(c->sm_count, OP_PART_ROWS / (MERGE_WARPS * MERGE_ROWS)), MERGE_WARPS * 32, 0, t.ws, t.o);
  return RPO_OK;
}

// 32-bit storage: BM rows of an item against tiles of keys on CUDA cores.
template <int DH, int BM>
static int chunk_f32(rpo_ctx* c, const PagedView<float>& view, const ChunkArgs& a, const float* q, int64_t q_stride, const float* k_new, const float* v_new,
                      int64_t new_stride, float scale, float* out, float* lse) {
  using Cfg = F32Cfg<DH, BM>;
  CUDA_TRY((allow_smem<paged_f32_kernel<DH, BM>>(c, Cfg::SMEM)));
  F32Args f;
  f.kv = view; f.c = a; f.q = q; f.q_stride = q_stride; f.scale_log2 = scale * 1.4426950408889634f;
  f.o.out = out; f.o.lse = lse; f.o.hq = a.hq; f.o.rep = a.hq / view.hkv; f.ws = split_ws(c, BM);
  f.tok = BM / f.o.rep;
  if ((int64_t)a.n_rows / f.tok + view.n_seqs > OP_MAX_ITEMS) return RPO_ERR_LIMIT;
  ChunkItem* items = (ChunkItem*)c->ws.op_items;
  ChunkPlan* plan = (ChunkPlan*)(items + OP_MAX_ITEMS);
  f.items = items; f.plan = plan;
  const int grid = std::min(Cfg::CTAS * c->sm_count, OP_GRID * c->sm_count);
  LAUNCH_OP(c, (chunk_prepare_kernel<float, DH, Cfg::BN / KV_BLOCK>), (prepare_grid<float, DH>(view, a, k_new)), 1024, view.n_seqs * 4, view, a, f.tok, grid, 2, 1, items,
            plan, k_new, v_new, new_stride);
  LAUNCH_OP(c, (paged_f32_kernel<DH, BM>), grid, 256, Cfg::SMEM, f);
  LAUNCH_OP(c, (split_merge_kernel<float, DH>), dim3(grid, BM == 64 ? BM / (MERGE_WARPS * MERGE_ROWS) : std::min(a.max_chunk * f.o.rep, BM)), MERGE_WARPS * 32, 0, f.ws, f.o);
  return RPO_OK;
}

template <typename T, int DH>
static int chunk_attention_t(rpo_ctx* c, const rpo_paged_kv* kv, const ChunkArgs& a, const void* q, int64_t q_stride, const void* k_new,
                             const void* v_new, int64_t new_stride, float scale, void* out, float* lse) {
  const PagedView<T> view = paged_view<T>(c, kv);
  const int64_t rows = a.max_chunk * (int64_t)(a.hq / kv->n_kv_heads);           // of the longest chunk, per KV head
  // Up to 16 rows have kernels of one 16-row tile.  16 bits: measured on both sides in paged_step.cuh.  32 bits, 32 sequences of
  // 1024 .. 4096, 12 on 2 heads of 128: 1 token 154 us (in 64-row tiles 227), 2 tokens 156 (233), 3 tokens 236 in 64-row tiles.
  if constexpr (std::is_same<T, bf16>::value) {
    if (rows <= StepCfg<DH>::ROWS)
      return chunk_steps<DH>(c, view, a, (const bf16*)q, q_stride, (const bf16*)k_new, (const bf16*)v_new, new_stride, scale, (bf16*)out, lse);
    return chunk_tiles<DH>(c, view, a, (const bf16*)q, q_stride, (const bf16*)k_new, (const bf16*)v_new, new_stride, scale, (bf16*)out, lse);
  } else {
    if (rows <= 16) return chunk_f32<DH, 16>(c, view, a, (const float*)q, q_stride, (const float*)k_new, (const float*)v_new, new_stride, scale, (float*)out, lse);
    return chunk_f32<DH, 64>(c, view, a, (const float*)q, q_stride, (const float*)k_new, (const float*)v_new, new_stride, scale, (float*)out, lse);
  }
}

extern "C" int rpo_chunk_attention(rpo_ctx* c, const rpo_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t max_chunk, const void* d_q,
                                   int64_t q_stride, const void* d_k_new, const void* d_v_new, int64_t kv_new_stride,
                                   const int32_t* d_q_offsets, const rpo_chunk_cfg* cfg, void* d_out, float* d_lse_out) {
  RPO_TRY(check_chunk(c, kv, n_rows, n_q_heads, max_chunk, d_q, q_stride, d_q_offsets, cfg));
  if ((n_rows > 0 && !d_out) || !aligned16(d_out) || !d_k_new != !d_v_new) return RPO_ERR_INVALID_ARG;
  if (d_k_new && (!aligned16(d_k_new) || !aligned16(d_v_new) || (kv_new_stride * (int64_t)c->esz) % 16 ||
                  (n_rows > 1 && kv_new_stride < (int64_t)kv->n_kv_heads * kv->head_dim)))
    return RPO_ERR_INVALID_ARG;
  if (n_rows == 0) return RPO_OK;
  RPO_TRY(enter(c));
  ProfScope ps(c, KC_ATTN);
  const ChunkArgs a = chunk_args(n_rows, n_q_heads, max_chunk, d_q_offsets, cfg);
#define CHUNK_ATTN(T, DH) chunk_attention_t<T, DH>(c, kv, a, d_q, q_stride, d_k_new, d_v_new, kv_new_stride, cfg->scale, d_out, d_lse_out)
  if (c->bf16) return kv->head_dim == 128 ? CHUNK_ATTN(bf16, 128) : CHUNK_ATTN(bf16, 64);
  return kv->head_dim == 128 ? CHUNK_ATTN(float, 128) : CHUNK_ATTN(float, 64);
#undef CHUNK_ATTN
}

template <int DH, int MT>
static int mass_steps(rpo_ctx* c, const PagedView<bf16>& view, const ChunkArgs& a, const bf16* q, int64_t q_stride, const float* lse, float scale,
                      const float* in, float* out, int stride) {
  using Cfg = MassStepCfg<DH, MT>;
  CUDA_TRY((allow_smem<mass_step_kernel<DH, MT>>(c, Cfg::SMEM + (OP_MAX_SEQS + 1) * 4)));
  MassArgs m;
  m.kv = view; m.c = a; m.q = q; m.q_stride = q_stride; m.scale_log2 = scale * 1.4426950408889634f; m.lse = lse; m.in = in; m.out = out;
  m.stride = stride; m.rep = a.hq / view.hkv;
  LAUNCH_OP(c, (mass_step_kernel<DH, MT>), 4 * c->sm_count, 128, Cfg::SMEM + (view.n_seqs + 1) * 4, m);
  return RPO_OK;
}

template <int DH>
static int mass_tiles(rpo_ctx* c, const PagedView<bf16>& view, const ChunkArgs& a, const bf16* q, int64_t q_stride, const float* lse, float scale,
                      const float* in, float* out, int stride) {
  using Cfg = MassCfg<DH>;
  CUDA_TRY((allow_smem<mass_chunk_kernel<DH>>(c, Cfg::SMEM)));
  MassTcArgs m;
  m.kv = view; m.c = a; m.scale_log2 = scale * 1.4426950408889634f; m.lse = lse; m.in = in; m.out = out; m.stride = stride;
  m.rep = a.hq / view.hkv; m.tq = MS_ROWS / m.rep;
  MassItem* items = (MassItem*)c->ws.op_items;
  ChunkPlan* plan = (ChunkPlan*)(items + OP_MAX_ITEMS);
  m.items = items; m.plan = plan; m.ws.part = c->ws.op_part_o; m.ws.rec = (SplitRec*)c->ws.op_rec;
  CUtensorMap qm, km;
  RPO_TRY(op_map_rows(c, &qm, q, q_stride, a.n_rows, a.hq, DH, m.rep, m.tq));
  RPO_TRY(op_map_pages(c, &km, view, view.k, DH));
  LAUNCH_OP(c, mass_plan_kernel, 1, 1024, view.n_seqs * 4, view, a, stride, m.tq, c->sm_count, 4, 2, items, plan);
  LAUNCH_OP(c, (mass_chunk_kernel<DH>), c->sm_count, Cfg::THREADS, Cfg::SMEM, qm, km, m);
  LAUNCH_OP(c, mass_merge_kernel, c->sm_count, MS_KEYS, 0, m.ws, in, out);
  return RPO_OK;
}

template <int DH, int BM>
static int mass_f32(rpo_ctx* c, const PagedView<float>& view, const ChunkArgs& a, const float* q, int64_t q_stride, const float* lse, float scale,
                    const float* in, float* out, int stride) {
  constexpr int smem = ((MF_KEYS + 2 * BM) * (DH + 4) + 2 * BM) * 4;
  CUDA_TRY((allow_smem<mass_f32_kernel<DH, BM>>(c, smem)));
  MassF32Args m;
  m.kv = view; m.c = a; m.q = q; m.q_stride = q_stride; m.scale_log2 = scale * 1.4426950408889634f; m.lse = lse; m.in = in; m.out = out;
  m.stride = stride; m.rep = a.hq / view.hkv;
  // every (sequence, KV head) has its CTAs, 16 per SM in all; they walk the key tiles there are, not those the table could hold
  const int tiles = ceil_div(std::min((int64_t)stride, (int64_t)view.table_stride * KV_BLOCK), MF_KEYS);
  const dim3 grid(std::min(tiles, ceil_div(16 * c->sm_count, (int64_t)view.hkv * view.n_seqs)), view.hkv, view.n_seqs);
  LAUNCH_OP(c, (mass_f32_kernel<DH, BM>), grid, 256, smem, m);
  return RPO_OK;
}

template <typename T, int DH>
static int attention_mass_t(rpo_ctx* c, const rpo_paged_kv* kv, const ChunkArgs& a, const void* q, int64_t q_stride, const float* lse, float scale,
                            const float* in, float* out, int stride) {
  const PagedView<T> view = paged_view<T>(c, kv);
  const int64_t rows = a.n_rows == 0 ? 0 : a.max_chunk * (int64_t)(a.hq / kv->n_kv_heads);
  // 16 bits, 128 sequences of 1024 .. 6144, 28 on 4 heads of 128: 1 token 104 us, 4 tokens (two 16-row tiles) 162, in the tiled
  // kernel 240 either way; 5 tokens there 242; 4 sequences of 100 .. 300, 12 on 2 heads: 12 us against 31.  32 bits, 32 sequences of
  // 1024 .. 4096, 12 on 2 heads of 128: 1 token 80 us (in 64-row tiles 137), 3 tokens 141 in 64-row tiles.
  if constexpr (std::is_same<T, bf16>::value) {
    if (rows <= 16) return mass_steps<DH, 1>(c, view, a, (const bf16*)q, q_stride, lse, scale, in, out, stride);
    if (rows <= 32) return mass_steps<DH, 2>(c, view, a, (const bf16*)q, q_stride, lse, scale, in, out, stride);
    return mass_tiles<DH>(c, view, a, (const bf16*)q, q_stride, lse, scale, in, out, stride);
  } else {
    if (rows <= 16) return mass_f32<DH, 16>(c, view, a, (const float*)q, q_stride, lse, scale, in, out, stride);
    return mass_f32<DH, 64>(c, view, a, (const float*)q, q_stride, lse, scale, in, out, stride);
  }
}

extern "C" int rpo_attention_mass(rpo_ctx* c, const rpo_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t max_chunk, const void* d_q,
                                  int64_t q_stride, const int32_t* d_q_offsets, const rpo_chunk_cfg* cfg, const float* d_lse,
                                  const float* d_mass_in, float* d_mass_out, int32_t mass_stride) {
  RPO_TRY(check_chunk(c, kv, n_rows, n_q_heads, max_chunk, d_q, q_stride, d_q_offsets, cfg));
  if ((n_rows > 0 && !d_lse) || !d_mass_out || mass_stride <= 0) return RPO_ERR_INVALID_ARG;
  if (kv->n_kv_heads > 65535) return RPO_ERR_LIMIT;
  RPO_TRY(enter(c));
  ProfScope ps(c, KC_ATTN);
  const ChunkArgs a = chunk_args(n_rows, n_q_heads, max_chunk, d_q_offsets, cfg);
#define ATTN_MASS(T, DH) attention_mass_t<T, DH>(c, kv, a, d_q, q_stride, d_lse, cfg->scale, d_mass_in, d_mass_out, mass_stride)
  if (c->bf16) return kv->head_dim == 128 ? ATTN_MASS(bf16, 128) : ATTN_MASS(bf16, 64);
  return kv->head_dim == 128 ? ATTN_MASS(float, 128) : ATTN_MASS(float, 64);
#undef ATTN_MASS
}

template <int THREADS, int KPT, int C>
static int evict_launch(rpo_ctx* c, EvictArgs a) {
  CUDA_TRY((allow_smem<evict_kernel<THREADS, KPT, C>>(c, (EV_MAX_STRIDE / 2 / 8 + 1) * 4)));
  a.list_cap = ceil_div(std::max(1, std::min(a.budget, a.mass_stride / 2 + 1)), C);     // holes: at most half of the slots
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.n_seqs * a.hkv * C); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = (size_t)a.list_cap * 4; cfg.stream = c->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = C > 1 ? 1 : 0;
  prof_begin(c, "evict_kernel");
  const cudaError_t e = cudaLaunchKernelEx(&cfg, evict_kernel<THREADS, KPT, C>, a);
  prof_end(c);
  c->launches++;
  CUDA_TRY(e);
  return RPO_OK;
}

extern "C" int rpo_evict_cache(rpo_ctx* c, const rpo_paged_kv* kv, const float* d_mass, const int32_t* d_positions, int32_t mass_stride,
                               int32_t budget, int32_t sinks, int32_t recent, int32_t* d_lens_out, int32_t* d_src_out, float* d_mass_out,
                               int32_t* d_positions_out, int32_t out_stride) {
  RPO_TRY(check_paged(c, kv));
  if (!d_mass || !d_positions || !d_lens_out || !d_src_out || !d_mass_out || !d_positions_out || mass_stride <= 0 || budget <= 0 ||
      sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget || out_stride < budget)
    return RPO_ERR_INVALID_ARG;
  if ((d_mass_out == d_mass || d_positions_out == d_positions) && out_stride != mass_stride) return RPO_ERR_INVALID_ARG;
  if (mass_stride > EV_MAX_STRIDE || (int64_t)kv->n_seqs * kv->n_kv_heads > 65535) return RPO_ERR_LIMIT;
  RPO_TRY(enter(c));
  EvictArgs a;
  a.lens = kv->d_lens; a.mass = d_mass; a.pos = d_positions; a.lens_out = d_lens_out; a.src = d_src_out; a.mass_out = d_mass_out;
  a.pos_out = d_positions_out; a.mass_stride = mass_stride; a.out_stride = out_stride; a.n_seqs = kv->n_seqs; a.hkv = kv->n_kv_heads;
  a.table_stride = kv->table_stride; a.budget = budget; a.sinks = sinks; a.recent = recent; a.status = c->d_status;
  a.k = (uint8_t*)kv->d_k; a.v = (uint8_t*)kv->d_v; a.table = kv->d_block_table; a.n_blocks = kv->n_blocks;
  a.row_bytes = kv->head_dim * (int)c->esz; a.head_bytes = (int64_t)kv->n_blocks * KV_BLOCK * a.row_bytes;
  a.write_lens = d_lens_out != kv->d_lens; a.list_cap = 0;
  // Registers hold 8 or 16 slots a thread; few slots take a small CTA, so that more (sequence, KV head)s run at once (four
  // CTAs of 256 or two of 512 threads fit an SM: 256 caches of up to 6144 slots took 90 us with 1024 threads).  A cluster is
  // as small as its registers hold the slots (236 caches of 13 315 slots: 387 us in clusters of eight, 49 us in one CTA
  // each), and grows while SMs would stay idle (32 caches of 3602: 37 us instead of 51).
  const int n = a.n_seqs * a.hkv;
  if (mass_stride <= 2048) {                                 // (a cluster for few small caches: 23 us instead of 12)
    RPO_TRY((evict_launch<256, 8, 1>(c, a)));
  } else {
    const int threads = mass_stride <= 8192 ? 512 : 1024;
    int cluster = 1;
    while (cluster < 8 && (mass_stride > cluster * threads * 16 || (int64_t)n * cluster * 2 <= c->sm_count)) cluster *= 2;
    if (mass_stride > 8 * 1024 * 16) RPO_TRY((evict_launch<1024, 0, 8>(c, a)));
    else if (threads == 512) RPO_TRY(cluster == 1 ? (evict_launch<512, 16, 1>(c, a)) : cluster == 2 ? (evict_launch<512, 16, 2>(c, a))
                                     : cluster == 4 ? (evict_launch<512, 16, 4>(c, a)) : (evict_launch<512, 16, 8>(c, a)));
    else RPO_TRY(cluster == 1 ? (evict_launch<1024, 16, 1>(c, a)) : cluster == 2 ? (evict_launch<1024, 16, 2>(c, a))
                 : cluster == 4 ? (evict_launch<1024, 16, 4>(c, a)) : (evict_launch<1024, 16, 8>(c, a)));
  }
  if (!a.write_lens) LAUNCH_OP(c, evict_lens_kernel, ceil_div(a.n_seqs, 256), 256, 0, a);
  return RPO_OK;
}
