// Entry points for rollouts with drafted tokens and shared pages (part of rpo_api.cu).
#pragma once

// One cluster per item (or one for all), launched plainly as the other operators on the caller's memory.
template <typename... KArgs, typename... Args>
static int launch_clusters(rpo_ctx* c, const char* label, void (*kern)(KArgs...), int ctas, int cluster, int threads, size_t smem, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = c->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  prof_begin(c, label);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, args...);
  prof_end(c);
  c->launches++;
  CUDA_TRY(e);
  return RPO_OK;
}

// Clusters of more than eight CTAs have to be asked for, once per device.
template <auto KERNEL>
static cudaError_t allow_large_clusters(rpo_ctx* c) {
  static OncePerDevice once;
  return once.run(c->device, [&] { return cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); });
}

template <int C>
static int verify_launch(rpo_ctx* c, VerifyArgs a, int n_seqs) {
  if (C > 8) CUDA_TRY((allow_large_clusters<verify_kernel<C>>(c)));
  CUDA_TRY((allow_smem<verify_kernel<C>>(c, VF_HIST + (((1 << 18) / C + 3) & ~3) * 4)));
  a.slice = (ceil_div(a.V, C) + 3) & ~3;
  return launch_clusters(c, "verify_kernel", verify_kernel<C>, n_seqs * C, C, VF_THREADS, (a.top_p24 < (1u << 24) ? VF_HIST : 0) + (size_t)a.slice * 4, a);
}

extern "C" int rpo_verify_drafts(rpo_ctx* c, int32_t n_seqs, int32_t n_rows, int32_t vocab, const float* d_logits, int64_t logits_stride,
                                 const float* d_draft_probs, int64_t probs_stride, const int32_t* d_tokens, const int32_t* d_parents,
                                 const int32_t* d_offsets, const float* d_uniform, const rpo_sampler* sampler, int32_t max_path, int32_t* d_path_out,
                                 int32_t* d_n_path_out, int32_t* d_next_out, float* d_logprobs_out) {
  if (!c || n_seqs < 0 || n_rows < 0 || vocab <= 0 || max_path <= 0 || !d_offsets || !d_path_out || !d_n_path_out || !d_next_out ||
      (n_rows > 0 && (!d_logits || !d_tokens || !d_parents || !d_uniform)) || logits_stride < vocab || (d_draft_probs && probs_stride < vocab))
    return RPO_ERR_INVALID_ARG;
  RPO_TRY(check_sampler(sampler));
  if (vocab >= (1 << 18) || n_seqs > (1 << 24)) return RPO_ERR_LIMIT;
  if (n_seqs == 0) return RPO_OK;
  RPO_TRY(enter(c));
  ProfScope ps(c, KC_SAMPLER);
  VerifyArgs a = {};
  a.logits = d_logits; a.logits_stride = logits_stride; a.probs = d_draft_probs; a.probs_stride = probs_stride;
  a.tokens = d_tokens; a.parents = d_parents; a.offsets = d_offsets; a.uniform = d_uniform;
  a.path = d_path_out; a.n_path = d_n_path_out; a.next = d_next_out; a.logprobs = d_logprobs_out;
  a.V = vocab; a.n_rows = n_rows; a.max_path = max_path; a.greedy = sampler->greedy != 0; a.eos_id = sampler->eos_id;
  a.temperature = sampler->temperature; a.top_p24 = (uint32_t)floorf(sampler->top_p * 16777216.0f); a.status = c->d_status;
  // Few sequences: clusters of sixteen (4 trees of 24 nodes over 151 936 tokens 32.9 us, clusters of eight 37.9; 8 chains of 9 with
  // probabilities 51, eight 59).  Many: eight, two of whose CTAs share an SM (16 such chains 80 us, sixteen 86; 128: 248 and 417).
  return n_seqs * 16 <= c->sm_count ? verify_launch<16>(c, a, n_seqs) : verify_launch<8>(c, a, n_seqs);
}

// All layers share pool size, tables and lengths; `l` describes their planes.
static int check_layers(rpo_ctx* c, const rpo_paged_kv* layers, int32_t n_layers, PageLayers* l) {
  if (!c || !layers || n_layers <= 0) return RPO_ERR_INVALID_ARG;
  if (n_layers > PG_MAX_LAYERS) return RPO_ERR_LIMIT;
  for (int i = 0; i < n_layers; ++i) {
    RPO_TRY(check_paged(c, layers + i));
    const rpo_paged_kv &x = layers[i], &y = layers[0];
    if (x.n_blocks != y.n_blocks || x.n_seqs != y.n_seqs || x.table_stride != y.table_stride || x.n_kv_heads != y.n_kv_heads || x.head_dim != y.head_dim ||
        x.d_block_table != y.d_block_table || x.d_lens != y.d_lens)
      return RPO_ERR_INVALID_ARG;
    l->k[i] = (uint8_t*)x.d_k; l->v[i] = (uint8_t*)x.d_v;
  }
  l->n_layers = n_layers; l->hkv = layers->n_kv_heads; l->n_blocks = layers->n_blocks; l->row_bytes = layers->head_dim * (int)c->esz;
  l->head_bytes = (int64_t)layers->n_blocks * KV_BLOCK * l->row_bytes;
  return layers->n_seqs > OP_MAX_SEQS ? RPO_ERR_LIMIT : RPO_OK;
}

static int check_pool(rpo_ctx* c, const rpo_page_pool* pool, const rpo_paged_kv* layers, int32_t n_layers, int n_items, PageLayers* l, PagePoolArgs* p) {
  if (!pool || !pool->d_refs || !pool->d_free || !pool->d_n_free || !pool->d_block_table || !pool->d_held) return RPO_ERR_INVALID_ARG;
  RPO_TRY(check_layers(c, layers, n_layers, l));
  if (pool->d_block_table != layers->d_block_table || pool->n_blocks != layers->n_blocks || pool->n_seqs != layers->n_seqs ||
      pool->table_stride != layers->table_stride)
    return RPO_ERR_INVALID_ARG;
  // a page's place among all that a call releases is a number below 2^29; so are pages and slots
  if (n_items > PG_MAX_ITEMS || (int64_t)std::max(n_items, 1) * pool->table_stride >= (1 << 29) || pool->table_stride >= (1 << 26)) return RPO_ERR_LIMIT;
  p->refs = pool->d_refs; p->free = pool->d_free; p->n_free = pool->d_n_free; p->table = pool->d_block_table; p->held = pool->d_held;
  p->n_blocks = pool->n_blocks; p->n_seqs = pool->n_seqs; p->stride = pool->table_stride; p->status = c->d_status;
  p->ws.copies = (PageCopy*)c->ws.op_pages; p->ws.counts = (int*)(p->ws.copies + PG_MAX_ITEMS); p->ws.ticket = p->ws.counts + PG_MAX_ITEMS;
  return RPO_OK;
}

static int page_cluster(int n_items) {
  int cluster = 1;
  while (cluster < PG_MAX_CLUSTER && n_items > cluster * PG_WARPS / 2) cluster *= 2;      // (half of the warps: their accesses spread over more SMs)
  return cluster;
}

// Planes that a CTA takes of each item: all SMs have work, and an item's look-ups are shared by eight planes at least.
static int planes_per_cta(const rpo_ctx* c, const PageLayers& l, int64_t items, int ctas_per_sm) {
  return (int)std::min<int64_t>(PG_PLANES, std::max<int64_t>(8, ceil_div(items * 2 * l.n_layers * l.hkv, ctas_per_sm * (int64_t)c->sm_count)));
}
static int plane_grid(const PageLayers& l, int64_t items, int per) { return (int)std::min<int64_t>(items * ceil_div(2 * (int64_t)l.n_layers * l.hkv, per), 1 << 20); }

static int copy_pages(rpo_ctx* c, const PageLayers& l, const PageWs& ws, int n, bool rare) {
  const int per = planes_per_cta(c, l, n, 8);
  const int grid = plane_grid(l, n, per);
  LAUNCH_OP(c, copy_pages_kernel, rare ? std::min(grid, 4 * c->sm_count) : grid, PG_MOVE_THREADS, 0, l, ws.copies, n, per, rare);
  return RPO_OK;
}

extern "C" int rpo_fork_pages(rpo_ctx* c, const rpo_page_pool* pool, const rpo_paged_kv* h_layers, int32_t n_layers, int32_t n_forks,
                              const int32_t* d_src, const int32_t* d_dst, const int32_t* d_fork_lens, int32_t* d_lens_out) {
  PageLayers l;
  ForkArgs a;
  if (n_forks < 0 || (n_forks > 0 && (!d_src || !d_dst || !d_fork_lens))) return RPO_ERR_INVALID_ARG;
  RPO_TRY(check_pool(c, pool, h_layers, n_layers, n_forks, &l, &a.p));
  if (n_forks == 0) return RPO_OK;
  RPO_TRY(enter(c));
  a.src = d_src; a.dst = d_dst; a.lens = d_fork_lens; a.lens_out = d_lens_out; a.n = n_forks;
  const int cluster = page_cluster(n_forks);
  RPO_TRY(launch_clusters(c, "fork_pages_kernel", fork_pages_kernel, cluster, cluster, PG_THREADS, 0, a));
  return copy_pages(c, l, a.p.ws, n_forks, false);
}

extern "C" int rpo_reserve_pages(rpo_ctx* c, const rpo_page_pool* pool, const rpo_paged_kv* h_layers, int32_t n_layers, const int32_t* d_lens,
                                 const int32_t* d_target_lens) {
  PageLayers l;
  ReserveArgs a;
  if (!d_lens || !d_target_lens) return RPO_ERR_INVALID_ARG;
  RPO_TRY(check_pool(c, pool, h_layers, n_layers, pool ? pool->n_seqs : 0, &l, &a.p));
  RPO_TRY(enter(c));
  a.lens = d_lens; a.target = d_target_lens;
  const int cluster = page_cluster(a.p.n_seqs);
  RPO_TRY(launch_clusters(c, "reserve_pages_kernel", reserve_pages_kernel, cluster, cluster, PG_THREADS, 0, a));
  return copy_pages(c, l, a.p.ws, a.p.n_seqs, true);
}

extern "C" int rpo_commit_path(rpo_ctx* c, const rpo_paged_kv* h_layers, int32_t n_layers, const int32_t* d_q_offsets, const int32_t* d_path,
                               int32_t path_stride, const int32_t* d_n_path, int32_t* d_lens_out) {
  PageLayers l;
  if (!d_q_offsets || !d_path || path_stride <= 0 || !d_n_path || !d_lens_out) return RPO_ERR_INVALID_ARG;
  RPO_TRY(check_layers(c, h_layers, n_layers, &l));
  RPO_TRY(enter(c));
  CommitArgs a;
  a.table = h_layers->d_block_table; a.lens = h_layers->d_lens; a.offsets = d_q_offsets; a.path = d_path; a.n_path = d_n_path; a.lens_out = d_lens_out;
  a.n_seqs = h_layers->n_seqs; a.stride = h_layers->table_stride; a.path_stride = path_stride; a.status = c->d_status;
  a.ticket = (int*)((PageCopy*)c->ws.op_pages + PG_MAX_ITEMS) + PG_MAX_ITEMS;
  const int per = planes_per_cta(c, l, a.n_seqs, 4);
  LAUNCH_OP(c, commit_path_kernel, plane_grid(l, a.n_seqs, per), PG_MOVE_THREADS, 0, l, a, per);
  return RPO_OK;
}
