// Attention of a chunk of new tokens over a caller-owned paged cache.
//   o_i = sum_j w_ij v_j,  w_ij = exp(scale q_i . k_j - lse_i),  lse_i = log sum_j exp(scale q_i . k_j)
// over the keys j visible to row i: j <= p_i, and with a window W also j > p_i - W or j < sinks.
#pragma once
#include "paged_kv.cuh"

namespace rpo {

// One warp per (row, query head): a lane scores one key of 32 at a time, then owns head_dim / 32 output dims.
template <typename T, int DH>
__global__ void __launch_bounds__(128) paged_attn_simple_kernel(PagedView<T> kv, ChunkArgs c, const T* __restrict__ q, int64_t q_stride,
                                                                float scale, T* __restrict__ out, float* __restrict__ lse_out) {
  constexpr int DPL = DH / 32;
  __shared__ float s_q[4][DH];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * 4 + warp;
  if (w >= (int64_t)c.n_rows * c.hq) return;
  const int row = (int)(w / c.hq), head = (int)(w % c.hq), h = head / (c.hq / kv.hkv);
  const int s = chunk_seq_of_row(c, kv.n_seqs, row);
  if (s < 0) return;
  const ChunkSpan sp = chunk_span(kv, c, s);
  if (row < sp.row0 || row >= sp.row0 + sp.rows) return;
  for (int d = lane; d < DH; d += 32) s_q[warp][d] = to_f32(q[row * q_stride + head * DH + d]);
  __syncwarp();
  const int p = sp.len - sp.rows + (row - sp.row0);
  float m = -INFINITY, l = 0.f, acc[DPL];
#pragma unroll
  for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
  for (int j0 = 0; j0 <= p; j0 += 32) {
    const int j = j0 + lane;
    const bool seen = chunk_visible(c, j, p);
    if (!__any_sync(0xffffffffu, seen)) continue;
    const int64_t at = seen ? paged_row<T, DH>(kv, s, j) : -1;
    float x = -INFINITY;
    if (at >= 0) {
      const T* kr = kv.k + h * kv.head_stride + at;
      x = 0.f;
      for (int d = 0; d < DH; ++d) x = fmaf(s_q[warp][d], to_f32(kr[d]), x);
      x *= scale;
    }
    const float mn = fmaxf(m, warp_max(x)), mu = mn == -INFINITY ? 0.f : mn;
    const float corr = expf(m - mu), e = expf(x - mu);
    l = l * corr + warp_sum(e);
#pragma unroll
    for (int i = 0; i < DPL; ++i) acc[i] *= corr;
    m = mn;
    for (int t = 0; t < 32; ++t) {
      const int64_t vt = __shfl_sync(0xffffffffu, at, t);
      const float et = __shfl_sync(0xffffffffu, e, t);
      if (vt < 0) continue;
      const T* vr = kv.v + h * kv.head_stride + vt;
#pragma unroll
      for (int i = 0; i < DPL; ++i) acc[i] = fmaf(et, to_f32(vr[i * 32 + lane]), acc[i]);
    }
  }
  const int64_t o = (int64_t)row * c.hq + head;
#pragma unroll
  for (int i = 0; i < DPL; ++i) out[o * DH + i * 32 + lane] = from_f32<T>(l > 0.f ? acc[i] / l : 0.f);
  if (lane == 0 && lse_out) lse_out[o] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace rpo
