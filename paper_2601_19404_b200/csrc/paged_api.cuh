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

constexpr int OP_MAX_SEQS = 4096, OP_MAX_REP = 64;

static int check_chunk(const rpo_ctx* c, const rpo_paged_kv* kv, int n_rows, int hq, int max_chunk, const void* d_q, int64_t q_stride,
                       const int32_t* d_q_offsets, const rpo_chunk_cfg* cfg) {
  RPO_TRY(check_paged(c, kv));
  if (n_rows < 0 || hq <= 0 || max_chunk <= 0 || !d_q || !d_q_offsets || !cfg || !(cfg->scale > 0.f) || std::isinf(cfg->scale) ||
      cfg->window < 0 || cfg->sinks < 0 || !aligned16(d_q) || (q_stride * (int64_t)c->esz) % 16)
    return RPO_ERR_INVALID_ARG;
  if (hq % kv->n_kv_heads || hq / kv->n_kv_heads > OP_MAX_REP) return RPO_ERR_SHAPE;
  if (n_rows > 1 && q_stride < (int64_t)hq * kv->head_dim) return RPO_ERR_INVALID_ARG;
  if (kv->n_seqs > OP_MAX_SEQS || (int64_t)n_rows * hq >= ((int64_t)1 << 30)) return RPO_ERR_LIMIT;
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
  a.offsets = offsets; a.n_rows = n_rows; a.max_chunk = max_chunk; a.window = cfg->window; a.sinks = cfg->sinks; a.hq = hq;
  return a;
}

template <typename T, int DH>
static int chunk_attention_t(rpo_ctx* c, const rpo_paged_kv* kv, const ChunkArgs& a, const void* q, int64_t q_stride, const void* k_new,
                             const void* v_new, int64_t new_stride, float scale, void* out, float* lse) {
  const PagedView<T> view = paged_view<T>(c, kv);
  if (k_new) {
    const int64_t n = (int64_t)a.n_rows * view.hkv * 2 * (DH * sizeof(T) / 16);
    LAUNCH_OP(c, (paged_append_kernel<T, DH>), grid_for(n, 256), 256, 0, view, a, (const T*)k_new, (const T*)v_new, new_stride);
  }
  LAUNCH_OP(c, (paged_attn_simple_kernel<T, DH>), ceil_div((int64_t)a.n_rows * a.hq, 4), 128, 0, view, a, (const T*)q, q_stride, scale, (T*)out, lse);
  return RPO_OK;
}

extern "C" int rpo_chunk_attention(rpo_ctx* c, const rpo_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t max_chunk, const void* d_q,
                                   int64_t q_stride, const void* d_k_new, const void* d_v_new, int64_t kv_new_stride,
                                   const int32_t* d_q_offsets, const rpo_chunk_cfg* cfg, void* d_out, float* d_lse_out) {
  RPO_TRY(check_chunk(c, kv, n_rows, n_q_heads, max_chunk, d_q, q_stride, d_q_offsets, cfg));
  if (!d_out || !aligned16(d_out) || !d_k_new != !d_v_new) return RPO_ERR_INVALID_ARG;
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

template <typename T, int DH>
static int attention_mass_t(rpo_ctx* c, const rpo_paged_kv* kv, const ChunkArgs& a, const void* q, int64_t q_stride, const float* lse, float scale,
                            const float* mass_in, float* mass_out, int mass_stride) {
  const PagedView<T> view = paged_view<T>(c, kv);
  const dim3 grid(ceil_div(std::min((int64_t)mass_stride, (int64_t)view.table_stride * KV_BLOCK), MASS_KEYS), view.hkv, view.n_seqs);
  LAUNCH_OP(c, (paged_mass_simple_kernel<T, DH>), grid, MASS_KEYS, 0, view, a, (const T*)q, q_stride, lse, scale, mass_in, mass_out, mass_stride);
  return RPO_OK;
}

extern "C" int rpo_attention_mass(rpo_ctx* c, const rpo_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t max_chunk, const void* d_q,
                                  int64_t q_stride, const int32_t* d_q_offsets, const rpo_chunk_cfg* cfg, const float* d_lse,
                                  const float* d_mass_in, float* d_mass_out, int32_t mass_stride) {
  RPO_TRY(check_chunk(c, kv, n_rows, n_q_heads, max_chunk, d_q, q_stride, d_q_offsets, cfg));
  if (!d_lse || !d_mass_out || mass_stride <= 0) return RPO_ERR_INVALID_ARG;
  if (kv->n_kv_heads > 65535) return RPO_ERR_LIMIT;
  RPO_TRY(enter(c));
  ProfScope ps(c, KC_ATTN);
  const ChunkArgs a = chunk_args(n_rows, n_q_heads, max_chunk, d_q_offsets, cfg);
#define ATTN_MASS(T, DH) attention_mass_t<T, DH>(c, kv, a, d_q, q_stride, d_lse, cfg->scale, d_mass_in, d_mass_out, mass_stride)
  if (c->bf16) return kv->head_dim == 128 ? ATTN_MASS(bf16, 128) : ATTN_MASS(bf16, 64);
  return kv->head_dim == 128 ? ATTN_MASS(float, 128) : ATTN_MASS(float, 64);
#undef ATTN_MASS
}

template <typename T, int DH>
static int evict_cache_t(rpo_ctx* c, const rpo_paged_kv* kv, const EvictArgs& a) {
  const size_t smem = evict_smem_bytes(a.mass_stride, a.budget);
  static bool attr_done[64] = {};
  if (tc_first_use_on_device(c, attr_done))
    CUDA_TRY(cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)evict_smem_bytes(EV_MAX_STRIDE, EV_MAX_STRIDE)));
  const int n = a.n_seqs * a.hkv;
  LAUNCH_OP(c, evict_select_kernel, n, EV_THREADS, smem, a);
  const dim3 grid(std::min(ceil_div(a.budget, 8), std::max(1, 148 * 16 / n)), n);
  LAUNCH_OP(c, (evict_move_kernel<T, DH>), grid, 256, 0, paged_view<T>(c, kv), a);
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
  if (c->bf16) return kv->head_dim == 128 ? evict_cache_t<bf16, 128>(c, kv, a) : evict_cache_t<bf16, 64>(c, kv, a);
  return kv->head_dim == 128 ? evict_cache_t<float, 128>(c, kv, a) : evict_cache_t<float, 64>(c, kv, a);
}
