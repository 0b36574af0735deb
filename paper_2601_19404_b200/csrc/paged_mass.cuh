// Attention weight that every cached key receives from a chunk of new tokens:
//   mass_out[s][h][j] = mass_in[s][h][j] + sum over rows i of the chunk and query heads of KV head h of
//                       exp(scale q_i . k_j - lse_i)        (keys j that row i sees)
// lse comes from the attention call.  One thread owns one key: sums run in row order, nothing is added atomically.
#pragma once
#include "paged_kv.cuh"

namespace rpo {

constexpr int MASS_KEYS = 128, MASS_ROWS = 32;

template <typename T, int DH>
__global__ void __launch_bounds__(MASS_KEYS) paged_mass_simple_kernel(PagedView<T> kv, ChunkArgs c, const T* __restrict__ q, int64_t q_stride,
                                                                      const float* __restrict__ lse, float scale, const float* __restrict__ mass_in,
                                                                      float* __restrict__ mass_out, int mass_stride) {
  __shared__ float s_q[MASS_ROWS][DH];
  __shared__ float s_lse[MASS_ROWS];
  __shared__ int s_pos[MASS_ROWS];
  const int s = blockIdx.z, h = blockIdx.y, rep = c.hq / kv.hkv;
  const ChunkSpan sp = chunk_span(kv, c, s);
  const int len = min(sp.len, mass_stride);
  const int key0 = blockIdx.x * MASS_KEYS, j = key0 + threadIdx.x;
  if (key0 >= len) return;
  float kr[DH];
  const int64_t at = j < len ? paged_row<T, DH>(kv, s, j) : -1;
#pragma unroll
  for (int d = 0; d < DH; ++d) kr[d] = at >= 0 ? to_f32(kv.k[h * kv.head_stride + at + d]) : 0.f;
  float sum = 0.f;
  const int n = sp.rows * rep;
  for (int r0 = 0; r0 < n; r0 += MASS_ROWS) {
    __syncthreads();
    for (int i = threadIdx.x; i < MASS_ROWS * DH; i += MASS_KEYS) {
      const int r = r0 + i / DH;
      s_q[i / DH][i % DH] = r < n ? to_f32(q[(sp.row0 + r / rep) * q_stride + (h * rep + r % rep) * DH + i % DH]) : 0.f;
    }
    if (threadIdx.x < MASS_ROWS) {
      const int r = r0 + threadIdx.x;
      s_lse[threadIdx.x] = r < n ? lse[(int64_t)(sp.row0 + r / rep) * c.hq + h * rep + r % rep] : 0.f;
      s_pos[threadIdx.x] = r < n ? sp.len - sp.rows + r / rep : -1;
    }
    __syncthreads();
    for (int r = 0; r < min(MASS_ROWS, n - r0); ++r) {
      if (at < 0 || !chunk_visible(c, j, s_pos[r])) continue;
      float x = 0.f;
#pragma unroll
      for (int d = 0; d < DH; ++d) x = fmaf(s_q[r][d], kr[d], x);
      sum += expf(x * scale - s_lse[r]);
    }
  }
  if (j < len) {
    const int64_t o = ((int64_t)s * kv.hkv + h) * mass_stride + j;
    mass_out[o] = (mass_in ? mass_in[o] : 0.f) + sum;
  }
}

}  // namespace rpo
