// Caller-owned paged KV cache of one layer: what the operators on it share.
//
//   K, V          [kv_head][block][16 tokens][head_dim] in the storage type, rows in plain order
//   block table   [sequence][table_stride]: the block of tokens 16 b .. 16 b + 15
//   lens          tokens of every sequence in the cache
//
// Nothing the device reads from the caller's arrays is trusted: lengths are clamped to what the table can name,
// chunk offsets to the rows there are, block ids to the pool (each sets a bit of the status word).
#pragma once
#include "kernels.cuh"

namespace rpo {

// Workspace of the operators: rows of the largest part of a split item (two parts per CTA), items of one call (2^18 full
// ones, and one more for every sequence, whose last may not be full).
constexpr int OP_GRID = 3;                // CTAs per SM at most in a kernel that leaves parts
constexpr int OP_MAX_SEQS = 4096;
constexpr int OP_PART_ROWS = 256, OP_MAX_ITEMS = (1 << 18) + OP_MAX_SEQS;
constexpr int STATUS_BAD_LENGTH = 8;      // a length, chunk offset or chunk size out of range (clamped)

template <typename T>
struct PagedView {
  T* k; T* v;
  const int32_t* table; const int32_t* lens;
  int64_t head_stride;                    // elements between the KV heads: n_blocks * 16 * head_dim
  int n_blocks, n_seqs, table_stride, hkv;
  int* status;
};

// Rows of the call that belong to sequence s, and the tokens it has in the cache (the chunk's included).
struct ChunkSpan { int row0, rows, len; };

struct ChunkArgs {
  const int32_t* offsets;                 // [n_seqs + 1]
  int n_rows, max_chunk, window, sinks;   // window 0: none
  int hq;
};

__device__ __forceinline__ int paged_len(const int32_t* lens, int s, int table_stride, int* status) {
  const int n = lens[s], most = table_stride * KV_BLOCK;
  if (n < 0 || n > most) { atomicOr(status, STATUS_BAD_LENGTH); return min(max(n, 0), most); }
  return n;
}

template <typename T>
__device__ __forceinline__ ChunkSpan chunk_span(const PagedView<T>& kv, const ChunkArgs& c, int s) {
  ChunkSpan sp;
  const int a = c.offsets[s], b = c.offsets[s + 1];
  sp.row0 = min(max(a, 0), c.n_rows);
  sp.rows = min(max(b - sp.row0, 0), min(c.max_chunk, c.n_rows - sp.row0));
  if (a < 0 || b < a || b > c.n_rows || b - a > c.max_chunk) atomicOr(kv.status, STATUS_BAD_LENGTH);
  sp.len = paged_len(kv.lens, s, kv.table_stride, kv.status);
  return sp;
}

// Sequence of a row: the last s with offsets[s] <= row (-1: the row is behind the last sequence).
__device__ __forceinline__ int chunk_seq_of_row(const ChunkArgs& c, int n_seqs, int row) {
  int lo = 0, hi = n_seqs;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (c.offsets[mid] <= row) lo = mid; else hi = mid - 1;
  }
  return lo < n_seqs ? lo : -1;
}

// Offset of a token's row inside one KV head, or -1 when the table names no block of the pool.
template <typename T, int DH>
__device__ __forceinline__ int64_t paged_row(const PagedView<T>& kv, int s, int token) {
  const int blk = kv.table[(int64_t)s * kv.table_stride + token / KV_BLOCK];
  if (blk < 0 || blk >= kv.n_blocks) { atomicOr(kv.status, STATUS_BAD_BLOCK); return -1; }
  return ((int64_t)blk * KV_BLOCK + token % KV_BLOCK) * DH;
}

// The chunk's K and V rows into their pages; 16 bytes per thread.  Token i of a chunk of n rows in a cache of len
// tokens lands at position len - n + i (rows whose position would be negative are dropped).
template <typename T, int DH>
__device__ __forceinline__ void paged_append(const PagedView<T>& kv, const ChunkArgs& c, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                             int64_t new_stride, int block, int n_blocks) {
  constexpr int EPC = 16 / sizeof(T), CPR = DH / EPC;        // elements per copy, copies per row
  const int64_t n = (int64_t)c.n_rows * kv.hkv * 2 * CPR;
  for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < n; i += (int64_t)n_blocks * blockDim.x) {
    const int ch = (int)(i % CPR);
    const int64_t j = i / CPR;
    const int h = (int)(j % kv.hkv), which = (int)((j / kv.hkv) & 1), row = (int)(j / (2 * kv.hkv));
    const int s = chunk_seq_of_row(c, kv.n_seqs, row);
    if (s < 0) continue;
    const ChunkSpan sp = chunk_span(kv, c, s);
    const int pos = sp.len - sp.rows + (row - sp.row0);
    if (row < sp.row0 || row >= sp.row0 + sp.rows || pos < 0) continue;
    const int64_t at = paged_row<T, DH>(kv, s, pos);
    if (at < 0) continue;
    const uint4 x = *reinterpret_cast<const uint4*>((which ? v_new : k_new) + row * new_stride + h * DH + ch * EPC);
    *reinterpret_cast<uint4*>((which ? kv.v : kv.k) + h * kv.head_stride + at + ch * EPC) = x;
  }
}

// Is key j visible to a query at position p?
__device__ __forceinline__ bool chunk_visible(const ChunkArgs& c, int j, int p) {
  return j <= p && (c.window <= 0 || j > p - c.window || j < c.sinks);
}

}  // namespace rpo
