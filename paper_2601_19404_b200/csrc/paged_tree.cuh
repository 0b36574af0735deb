// Chunks that are trees of drafted tokens: which of the chunk's slots a node sees.
//
// Node i of a sequence's n nodes lies in slot past + i of its cache (past = len - n cached tokens) and names its parent, a
// node before it, or -1: the last cached token.  Its position is past + depth.  It sees the cached tokens as any token at that
// position does, and of the tree's slots itself and its ancestors, under a window the last `window` of them and those at
// positions below `sinks`.  A node whose chain of parents does not end at -1 is no node: it sees nothing, is seen by none,
// and its K and V are not written.
//
// Attention differs from that of causal chunks in the mask of the chunk's own slots alone.  Up to 16 rows (paged_step.cuh) and in
// 32 bits (paged_f32.cuh) it runs in the same kernels with one more template parameter; paged_treetile.cuh holds the 16-bit kernel
// of larger trees.  Up to 16 rows the warp that works on an item finds the masks with shuffles; the others read them from a list
// that tree_rows below writes, one bit per slot.
#pragma once
#include "paged_kv.cuh"

namespace rpo {

constexpr int TREE_MAX_NODES = 256, TREE_WORDS = TREE_MAX_NODES / 32, TREE_MAX_ROWS = 1 << 17;

struct TreeRow { uint32_t seen[TREE_WORDS]; int depth, pad[3]; };       // depth -1: no node

// The parent of node i, -2 where there is no node.
__device__ __forceinline__ int tree_parent(const ChunkArgs& c, const ChunkSpan& sp, int past, int i, int* status) {
  const int p = c.parents[sp.row0 + i];
  if (p >= i || p < -2 || past + i < 0) { atomicOr(status, STATUS_BAD_LENGTH); return -2; }
  return p;
}

// Is an ancestor `up` steps above a node of this depth inside its window?
__device__ __forceinline__ bool tree_in_window(const ChunkArgs& c, int past, int depth, int up) {
  return c.window <= 0 || up < c.window || past + depth - up < c.sinks;
}

// A sequence of at most 16 nodes, node i in lane i.
struct TreeLane { uint32_t seen, nodes; int depth; };

__device__ __forceinline__ TreeLane tree_lane(const ChunkArgs& c, const ChunkSpan& sp, int past, int lane, int* status) {
  TreeLane t;
  const int parent = lane < min(sp.rows, 16) ? tree_parent(c, sp, past, lane, status) : -2;
  t.depth = 0;
  int j = parent;
  while (__any_sync(0xffffffffu, j >= 0)) {
    const int above = __shfl_sync(0xffffffffu, parent, max(j, 0));
    if (j >= 0) { ++t.depth; j = above; }
  }
  const bool node = j == -1;
  t.nodes = __ballot_sync(0xffffffffu, node);
  t.seen = node ? 1u << lane : 0u;
  j = node ? parent : -1;
  for (int up = 1; __any_sync(0xffffffffu, j >= 0); ++up) {
    const int above = __shfl_sync(0xffffffffu, parent, max(j, 0));
    if (j >= 0) {
      if (tree_in_window(c, past, t.depth, up)) t.seen |= 1u << j;
      j = above;
    }
  }
  return t;
}

// Masks and depths of a sequence's nodes, found by all threads of a CTA; `s_parent` keeps the parents, s_depth the depths.
struct TreeShared { int parent[TREE_MAX_NODES], depth[TREE_MAX_NODES]; uint32_t seen[TREE_MAX_NODES][TREE_WORDS + 1]; };

__device__ __forceinline__ void tree_rows(const ChunkArgs& c, const ChunkSpan& sp, int past, TreeShared& sh, bool write, int* status) {
  const int n = min(sp.rows, TREE_MAX_NODES);
  for (int i = threadIdx.x; i < n; i += blockDim.x) sh.parent[i] = tree_parent(c, sp, past, i, status);
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    int depth = 0, j = i;
    while (sh.parent[j] >= 0) { j = sh.parent[j]; ++depth; }
    if (sh.parent[j] != -1) depth = -1;
    sh.depth[i] = depth;
    if (!write) continue;
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) sh.seen[i][w] = 0;
    if (depth >= 0)
      for (int up = 0, k = i; k >= 0; ++up, k = sh.parent[k])
        if (tree_in_window(c, past, depth, up)) sh.seen[i][k >> 5] |= 1u << (k & 31);
    TreeRow row;
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) row.seen[w] = sh.seen[i][w];
    row.depth = depth; row.pad[0] = row.pad[1] = row.pad[2] = 0;
    c.tree[sp.row0 + i] = row;
  }
  __syncthreads();
}

// 64 bits of a row's mask from slot `from` of the chunk on (-63 .. ; slots outside are not seen).
__device__ __forceinline__ uint64_t tree_bits(const uint32_t* seen, int from) {
  if (from < 0) return from <= -64 ? 0ull : (((uint64_t)seen[1] << 32) | seen[0]) << -from;
  const int w = from >> 5, s = from & 31;
  const uint32_t x0 = w < TREE_WORDS ? seen[w] : 0, x1 = w + 1 < TREE_WORDS ? seen[w + 1] : 0, x2 = w + 2 < TREE_WORDS ? seen[w + 2] : 0;
  return ((uint64_t)__funnelshift_r(x1, x2, s) << 32) | __funnelshift_r(x0, x1, s);
}

// The nodes' K and V into their slots, by the `block`-th of n_blocks CTAs of a sequence.
template <typename T, int DH>
__device__ __forceinline__ void tree_append(const PagedView<T>& kv, int s, const ChunkSpan& sp, int past, const TreeShared& sh, const T* __restrict__ k_new,
                                            const T* __restrict__ v_new, int64_t new_stride, int block, int n_blocks) {
  constexpr int EPC = 16 / sizeof(T), CPR = DH / EPC;
  const int n = min(sp.rows, TREE_MAX_NODES) * kv.hkv * 2 * CPR;
  for (int x = block * blockDim.x + threadIdx.x; x < n; x += n_blocks * blockDim.x) {
    const int ch = x % CPR, h = (x / CPR) % kv.hkv, which = (x / CPR / kv.hkv) & 1, i = x / CPR / kv.hkv / 2;
    if (sh.depth[i] < 0) continue;
    const int64_t at = paged_row<T, DH>(kv, s, past + i);
    if (at < 0) continue;
    const uint4 y = *reinterpret_cast<const uint4*>((which ? v_new : k_new) + (int64_t)(sp.row0 + i) * new_stride + h * DH + ch * EPC);
    *reinterpret_cast<uint4*>((which ? kv.v : kv.k) + h * kv.head_stride + at + ch * EPC) = y;
  }
}

}  // namespace rpo
