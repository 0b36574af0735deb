// Pages of a caller-owned cache under reference counts: sequences that become the first tokens of others (fork), take or give
// back pages (reserve), and keep the accepted nodes of a tree of drafted tokens (commit).
//
// Bound by latency where little is copied (a few dependent look-ups and barriers), by HBM where much is (the copied rows
// once each way).  Fork and reserve change tables, counts and the stack of free pages in one cluster, whose barriers order the
// phases, and leave a list of pages to copy; a second kernel copies those in all layers, a warp per page and plane (a plane
// is K or V of one KV head of one layer) with eight 16-byte pieces per lane in flight.  Which page goes where is a
// matter of the order of forks or sequences alone, never of timing:
//   taken    the k-th page that the call needs, in order of (fork or sequence, page of it), is free[n_free - 1 - k]
//   released a page whose count falls to 0 is pushed once, at the place of the first (fork or sequence, page) that drops it
#pragma once
#include <climits>

#include "attn_tc.cuh"
#include "paged_chunk.cuh"
#include "paged_kv.cuh"

namespace rpo {

constexpr int STATUS_NO_PAGES = 16;       // fewer free pages than a call needs
constexpr int PG_MAX_LAYERS = 128, PG_MAX_ITEMS = OP_MAX_SEQS;
constexpr int PG_THREADS = 1024, PG_WARPS = PG_THREADS / 32, PG_MAX_CLUSTER = 8;
constexpr int PG_PER_THREAD = PG_MAX_ITEMS / PG_THREADS;
constexpr int PG_MARK = 1 << 30;          // on a table entry during a call: this page is replaced by one of the sequence's own
constexpr int PG_CLAIM = -(1 << 30);      // count of a page that nobody holds, plus the place of the first to drop it

struct PageLayers {                       // all layers of a cache: same pool, tables and head layout
  uint8_t *k[PG_MAX_LAYERS], *v[PG_MAX_LAYERS];
  int64_t head_bytes;
  int n_layers, hkv, row_bytes, n_blocks;
  __device__ __forceinline__ int planes() const { return 2 * n_layers * hkv; }
  __device__ __forceinline__ uint8_t* plane(int p) const {
    const int h = p % hkv, l = p / hkv;
    return ((l & 1) ? v[l >> 1] : k[l >> 1]) + h * head_bytes;
  }
};

struct PageCopy { int from, to, rows, pad; };            // rows 0: nothing to copy

struct PageWs { PageCopy* copies; int *counts, *ticket; };      // [PG_MAX_ITEMS], [PG_MAX_ITEMS], one (zero between calls)

struct PagePoolArgs {
  int32_t *refs, *free, *n_free, *table, *held;
  int n_blocks, n_seqs, stride;
  int* status;
  PageWs ws;
  __device__ __forceinline__ void bad_length() const { atomicOr(status, STATUS_BAD_LENGTH); }
  __device__ __forceinline__ int clamped(int n, int most) const {
    if (n < 0 || n > most) { bad_length(); return min(max(n, 0), most); }
    return n;
  }
  __device__ __forceinline__ int pages_held(int s) const { return clamped(held[s], stride); }
  __device__ __forceinline__ int free_pages() const { return clamped(*n_free, n_blocks); }
  __device__ __forceinline__ bool in_pool(int page) const {
    if (page >= 0 && page < n_blocks) return true;
    atomicOr(status, STATUS_BAD_BLOCK);
    return false;
  }
  __device__ __forceinline__ int count_of(int page) const { return *(volatile int*)(refs + page); }
};

struct ForkArgs { PagePoolArgs p; const int32_t *src, *dst, *lens; int32_t* lens_out; int n; };
struct ReserveArgs { PagePoolArgs p; const int32_t *lens, *target; };

struct PageShared { int64_t scan[32]; int first[PG_MAX_ITEMS + 1], taken; };   // first: pages needed, then released, before item i

// sh.first[i] = sum of count(i') over i' < i, for i <= n; all threads of the CTA.
template <typename F>
__device__ __forceinline__ void page_prefix(int n, PageShared& sh, F count) {
  const int per = (n + PG_THREADS - 1) / PG_THREADS, i0 = threadIdx.x * per;
  int c[PG_PER_THREAD], sum = 0;
#pragma unroll
  for (int k = 0; k < PG_PER_THREAD; ++k) {
    c[k] = k < per && i0 + k < n ? count(i0 + k) : 0;
    sum += c[k];
  }
  int64_t before, all;
  plan_scan(sum, before, all, sh.scan);
#pragma unroll
  for (int k = 0; k < PG_PER_THREAD; ++k) {
    if (k < per && i0 + k < n) sh.first[i0 + k] = (int)before;
    before += c[k];
  }
  if (threadIdx.x == 0) sh.first[n] = (int)all;
  __syncthreads();
}

// Items are served in order as long as the free pages last; those that need none always are.
__device__ __forceinline__ bool page_served(const PagePoolArgs& p, const PageShared& sh, int i, int n_free) {
  if (sh.first[i + 1] <= n_free || sh.first[i + 1] == sh.first[i]) return true;
  atomicOr(p.status, STATUS_NO_PAGES);
  return false;
}
__device__ __forceinline__ int page_taken(PageShared& sh, int n, int n_free) {          // pages that the served ones take
  if (threadIdx.x == 0) sh.taken = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += PG_THREADS) if (sh.first[i + 1] <= n_free) atomicMax(&sh.taken, sh.first[i + 1]);
  __syncthreads();
  return sh.taken;
}

// One bit for each of a warp's items i = warp, warp + warps, ...
struct ItemBits {
  uint32_t x[PG_MAX_ITEMS / PG_WARPS / 32] = {};
  __device__ __forceinline__ void set(int k) {
#pragma unroll
    for (int w = 0; w < PG_MAX_ITEMS / PG_WARPS / 32; ++w) if (k >> 5 == w) x[w] |= 1u << (k & 31);
  }
  __device__ __forceinline__ bool get(int k) const {
    uint32_t y = 0;
#pragma unroll
    for (int w = 0; w < PG_MAX_ITEMS / PG_WARPS / 32; ++w) if (k >> 5 == w) y = x[w];
    return (y >> (k & 31)) & 1;
  }
};

// f(slot, page) for the slots [lo, hi) of a table row, 32 at a time, one per lane; page -1: no slot, or none of the pool.
// MARKS: entries may carry PG_MARK.
template <bool MARKS = false, typename F>
__device__ __forceinline__ void page_slots(const PagePoolArgs& p, int s, int lo, int hi, F f) {
  const int lane = threadIdx.x & 31;
  int32_t* row = p.table + (int64_t)s * p.stride;
  for (int j = lo; j < hi; j += 32) {
    int page = -1;
    if (j + lane < hi) { page = row[j + lane]; if (!p.in_pool(MARKS ? page & ~PG_MARK : page)) page = -1; }
    f(j + lane, page);
  }
}

// The releasing half of a call.  dropped(i, f) calls f(slot, page) for the pages that item i gives up, slots ascending, a
// warp together (page -1: none in this lane); finish(i) runs last, when the item's old table row is not needed any more.
template <typename D, typename F>
__device__ __forceinline__ void page_release(const PagePoolArgs& p, int n, int n_free, int n_taken, PageShared& sh, D dropped, F finish) {
  const int lane = threadIdx.x & 31, warp = blockIdx.x * PG_WARPS + (threadIdx.x >> 5), warps = gridDim.x * PG_WARPS;
  fa::cluster_sync();                                    // counts grow before they fall
  for (int i = warp; i < n; i += warps) dropped(i, [&](int, int page) { if (page >= 0) atomicSub(p.refs + page, 1); });
  fa::cluster_sync();
  for (int i = warp; i < n; i += warps)
    dropped(i, [&](int slot, int page) {
      if (page < 0) return;
      const int r = p.count_of(page);
      if (r == 0 || r < PG_CLAIM / 2) atomicMin(p.refs + page, PG_CLAIM + i * p.stride + slot);
    });
  fa::cluster_sync();
  auto claimed = [&](int i, int slot, int page) { return page >= 0 && p.count_of(page) == PG_CLAIM + i * p.stride + slot; };
  for (int i = warp; i < n; i += warps) {
    int c = 0;
    dropped(i, [&](int slot, int page) { c += __popc(__ballot_sync(0xffffffffu, claimed(i, slot, page))); });
    if (lane == 0) p.ws.counts[i] = c;
  }
  fa::cluster_sync();
  page_prefix(n, sh, [&](int i) { return *(volatile int*)(p.ws.counts + i); });
  const int base = n_free - n_taken;
  for (int i = warp; i < n; i += warps) {
    int at = base + sh.first[i];
    if (sh.first[i + 1] > sh.first[i])
      dropped(i, [&](int slot, int page) {
        const bool mine = claimed(i, slot, page);
        const unsigned who = __ballot_sync(0xffffffffu, mine);
        const int to = at + __popc(who & ((1u << lane) - 1));
        if (mine) {
          p.refs[page] = 0;
          if (to < p.n_blocks) p.free[to] = page; else p.bad_length();
        }
        at += __popc(who);
      });
    __syncwarp();
    finish(i);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.n_free = min(base + sh.first[n], p.n_blocks);
}

__global__ void __launch_bounds__(PG_THREADS) fork_pages_kernel(ForkArgs a) {
  const PagePoolArgs& p = a.p;
  __shared__ PageShared sh;
  __shared__ int s_dst[PG_MAX_ITEMS];                    // first fork that writes to a sequence
  const int tid = threadIdx.x, lane = tid & 31, warp = blockIdx.x * PG_WARPS + (tid >> 5), warps = gridDim.x * PG_WARPS;
  const int n_free = p.free_pages();
  for (int s = tid; s < p.n_seqs; s += PG_THREADS) s_dst[s] = INT_MAX;
  __syncthreads();
  for (int i = tid; i < a.n; i += PG_THREADS) { const int d = a.dst[i]; if (d >= 0 && d < p.n_seqs) atomicMin(s_dst + d, i); }
  __syncthreads();
  auto valid = [&](int i) {
    const int d = a.dst[i], s = a.src[i], len = a.lens[i];
    return d >= 0 && d < p.n_seqs && s >= 0 && s < p.n_seqs && s_dst[d] == i && s_dst[s] == INT_MAX && len >= 0 && len <= p.pages_held(s) * KV_BLOCK;
  };
  page_prefix(a.n, sh, [&](int i) {
    const bool ok = valid(i);
    if (!ok) p.bad_length();
    return ok && a.lens[i] % KV_BLOCK ? 1 : 0;
  });
  const int n_taken = page_taken(sh, a.n, n_free);
  ItemBits ok;
  for (int i = warp, k = 0; i < a.n; i += warps, ++k) {
    PageCopy copy = {-1, -1, 0, 0};
    if (valid(i) && page_served(p, sh, i, n_free)) {
      ok.set(k);
      const int len = a.lens[i], whole = len / KV_BLOCK, s = a.src[i];
      page_slots(p, s, 0, whole, [&](int, int page) { if (page >= 0) atomicAdd(p.refs + page, 1); });
      if (len % KV_BLOCK) {
        copy.from = p.table[(int64_t)s * p.stride + whole];
        copy.to = p.free[n_free - 1 - sh.first[i]];
        if (!p.in_pool(copy.to)) copy.to = -1;
        if (p.in_pool(copy.from) && copy.to >= 0) copy.rows = len % KV_BLOCK;
        if (lane == 0 && copy.to >= 0) p.refs[copy.to] = 1;
      }
    }
    if (lane == 0) p.ws.copies[i] = copy;
  }
  page_release(p, a.n, n_free, n_taken, sh,
               [&](int i, auto f) { if (ok.get((i - warp) / warps)) page_slots(p, a.dst[i], 0, p.pages_held(a.dst[i]), f); },
               [&](int i) {
                 if (!ok.get((i - warp) / warps)) return;
                 const int len = a.lens[i], whole = len / KV_BLOCK, part = len % KV_BLOCK ? 1 : 0;
                 const int32_t* from = p.table + (int64_t)a.src[i] * p.stride;
                 int32_t* to = p.table + (int64_t)a.dst[i] * p.stride;
                 for (int j = lane; j < whole; j += 32) to[j] = from[j];
                 if (lane == 0) {
                   if (part) to[whole] = p.ws.copies[i].to;
                   p.held[a.dst[i]] = whole + part;
                   if (a.lens_out) a.lens_out[a.dst[i]] = len;
                 }
               });
}

// A page that is replaced: its table entry becomes the new page with PG_MARK until the old one is released; the old one's
// number waits in the new one's count, which nobody else looks at before.
constexpr int PG_OLD = PG_CLAIM / 2;

struct ReserveSeq { int held, len, want; };

__global__ void __launch_bounds__(PG_THREADS) reserve_pages_kernel(ReserveArgs a) {
  const PagePoolArgs& p = a.p;
  __shared__ PageShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = blockIdx.x * PG_WARPS + (tid >> 5), warps = gridDim.x * PG_WARPS;
  const int n_free = p.free_pages(), n = p.n_seqs, most = p.stride * KV_BLOCK;
  auto seq = [&](int s) {
    ReserveSeq x;
    x.held = p.pages_held(s);
    const int target = p.clamped(a.target[s], most);
    x.len = p.clamped(min(p.clamped(a.lens[s], most), target), x.held * KV_BLOCK);
    x.want = (target + KV_BLOCK - 1) / KV_BLOCK;
    return x;
  };
  for (int s = warp; s < n; s += warps) {
    const ReserveSeq x = seq(s);
    int32_t* row = p.table + (int64_t)s * p.stride;
    int need = max(0, x.want - x.held);
    page_slots(p, s, x.len / KV_BLOCK, min(x.held, x.want), [&](int slot, int page) {
      const bool others = page >= 0 && p.count_of(page) > 1;
      if (others) row[slot] = page | PG_MARK;
      else if (page < 0 && slot < min(x.held, x.want) && row[slot] >= 0) row[slot] = -1;      // (a number that could pass for a mark)
      need += __popc(__ballot_sync(0xffffffffu, others));
    });
    if (lane == 0) p.ws.counts[s] = need;
  }
  fa::cluster_sync();
  page_prefix(n, sh, [&](int s) { return *(volatile int*)(p.ws.counts + s); });
  const int n_taken = page_taken(sh, n, n_free);
  ItemBits ok;
  for (int s = warp, k = 0; s < n; s += warps, ++k) {
    const ReserveSeq x = seq(s);
    int32_t* row = p.table + (int64_t)s * p.stride;
    const bool served = page_served(p, sh, s, n_free);
    if (served) ok.set(k);
    PageCopy copy = {-1, -1, 0, 0};
    int at = n_free - 1 - sh.first[s];
    const int lo = x.len / KV_BLOCK, shared_end = min(x.held, x.want);
    for (int j = lo; j < (served ? x.want : shared_end); j += 32) {
      const int slot = j + lane, entry = slot < shared_end ? row[slot] : 0;
      const bool marked = slot < shared_end && entry >= 0 && (entry & PG_MARK);
      const bool fresh = served && (marked || (slot >= x.held && slot < x.want));
      const unsigned who = __ballot_sync(0xffffffffu, fresh);
      int page = fresh ? p.free[max(0, at - __popc(who & ((1u << lane) - 1)))] : -1;
      if (fresh && !p.in_pool(page)) page = -1;
      at -= __popc(who);
      if (marked) {
        const int old = entry & ~PG_MARK;
        row[slot] = page >= 0 ? page | PG_MARK : old;
        if (page >= 0) p.refs[page] = PG_OLD + old;
        if (page >= 0 && slot == lo && x.len % KV_BLOCK) copy = PageCopy{old, page, x.len % KV_BLOCK, 0};
      } else if (fresh) {
        row[slot] = page;
        if (page >= 0) p.refs[page] = 1;
      }
    }
    if (lane == 0) p.ws.copies[s] = copy;                  // (slot lo is lane 0's)
  }
  page_release(p, n, n_free, n_taken, sh,
               [&](int s, auto f) {
                 if (!ok.get((s - warp) / warps)) return;
                 const ReserveSeq x = seq(s);
                 page_slots<true>(p, s, x.len / KV_BLOCK, x.held, [&](int slot, int page) {
                   int old = -1;
                   if (page >= 0 && (page & PG_MARK)) {
                     old = p.count_of(page & ~PG_MARK) - PG_OLD;
                     if (old < 0 || old >= p.n_blocks) old = -1;
                   } else if (slot >= x.want) old = page;
                   f(slot, old);
                 });
               },
               [&](int s) {
                 if (!ok.get((s - warp) / warps)) return;
                 const ReserveSeq x = seq(s);
                 page_slots<true>(p, s, x.len / KV_BLOCK, min(x.held, x.want), [&](int slot, int page) {
                   if (page < 0 || !(page & PG_MARK)) return;
                   p.table[(int64_t)s * p.stride + slot] = page & ~PG_MARK;
                   p.refs[page & ~PG_MARK] = 1;
                 });
                 __syncwarp();
                 if (lane == 0) p.held[s] = x.want;
               });
}

// The first rows of pages, in every plane.
constexpr int PG_LOADS = 8;

__global__ void __launch_bounds__(256) copy_pages_kernel(const __grid_constant__ PageLayers l, const PageCopy* copies, int n) {
  const int lane = threadIdx.x & 31, planes = l.planes();
  const int64_t total = (int64_t)n * planes, warps = (int64_t)gridDim.x * 8;
  for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < total; w += warps) {
    const PageCopy c = copies[w / planes];
    if (c.rows == 0) continue;
    uint8_t* base = l.plane((int)(w % planes));
    const int64_t page_bytes = (int64_t)KV_BLOCK * l.row_bytes;
    const uint4* from = reinterpret_cast<const uint4*>(base + c.from * page_bytes);
    uint4* to = reinterpret_cast<uint4*>(base + c.to * page_bytes);
    const int pieces = c.rows * l.row_bytes / 16;
    for (int i0 = lane; i0 < pieces; i0 += 32 * PG_LOADS) {
      uint4 x[PG_LOADS];
#pragma unroll
      for (int u = 0; u < PG_LOADS; ++u) if (i0 + 32 * u < pieces) x[u] = from[i0 + 32 * u];
#pragma unroll
      for (int u = 0; u < PG_LOADS; ++u) if (i0 + 32 * u < pieces) to[i0 + 32 * u] = x[u];
    }
  }
}

// Commit: the rows of the accepted nodes, in ascending order, to the front of the tree's slots.  A warp moves those of one
// sequence and plane in order, PG_LOADS pieces per lane at once; a row's source never lies before its destination, so what
// is read later has not been overwritten.  The CTA that ends last writes the lengths, which the others have read.
struct CommitArgs {
  const int32_t *table, *lens, *offsets, *path, *n_path; int32_t* lens_out;
  int n_seqs, stride, path_stride;
  int *status, *ticket;
};

struct CommitSeq { int past, n, len; };                  // n < 0: left alone

__device__ __forceinline__ CommitSeq commit_seq(const CommitArgs& a, int s) {      // by a whole warp
  const int lane = threadIdx.x & 31;
  CommitSeq x;
  x.len = paged_len(a.lens, s, a.stride, a.status);
  const int o0 = a.offsets[s], o1 = a.offsets[s + 1], n = a.n_path[s];
  const int64_t rows = (int64_t)o1 - o0;
  x.past = x.len - (int)min(max(rows, (int64_t)0), (int64_t)x.len);
  bool ok = rows >= 0 && rows <= x.len && n >= 0 && n <= a.path_stride && n <= rows;
  if (ok)
    for (int i = lane; i < n; i += 32) {
      const int32_t* path = a.path + (int64_t)s * a.path_stride;
      const int to = path[i];
      if (to < i || to >= rows || (i > 0 && to <= path[i - 1])) ok = false;
    }
  ok = __all_sync(0xffffffffu, ok);
  if (!ok && lane == 0) atomicOr(a.status, STATUS_BAD_LENGTH);
  x.n = ok ? n : -1;
  return x;
}

__global__ void __launch_bounds__(256) commit_path_kernel(const __grid_constant__ PageLayers l, CommitArgs a) {
  __shared__ int s_last;
  const int lane = threadIdx.x & 31, planes = l.planes(), lanes = l.row_bytes / 16, per = 32 / lanes;      // lanes of a row, rows at once
  const int64_t total = (int64_t)a.n_seqs * planes, warps = (int64_t)gridDim.x * 8;
  for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < total; w += warps) {
    const int s = (int)(w / planes);
    const CommitSeq q = commit_seq(a, s);
    if (q.n <= 0) continue;
    uint8_t* base = l.plane((int)(w % planes)) + (lane % lanes) * 16;
    const int32_t* path = a.path + (int64_t)s * a.path_stride;
    const int32_t* row = a.table + (int64_t)s * a.stride;
    auto place = [&](int slot) -> int64_t {
      const int page = row[slot / KV_BLOCK];
      if (page < 0 || page >= l.n_blocks) { atomicOr(a.status, STATUS_BAD_BLOCK); return -1; }
      return ((int64_t)page * KV_BLOCK + slot % KV_BLOCK) * l.row_bytes;
    };
    for (int i0 = lane / lanes; i0 - lane / lanes < q.n; i0 += per * PG_LOADS) {
      uint4 x[PG_LOADS];
      int64_t to[PG_LOADS];
#pragma unroll
      for (int u = 0; u < PG_LOADS; ++u) {
        const int i = i0 + per * u, node = i < q.n ? path[i] : i;
        to[u] = -1;
        if (node != i) {
          const int64_t from = place(q.past + node);
          to[u] = place(q.past + i);
          if (from < 0) to[u] = -1; else x[u] = *reinterpret_cast<const uint4*>(base + from);
        }
      }
      __syncwarp();
#pragma unroll
      for (int u = 0; u < PG_LOADS; ++u) if (to[u] >= 0) *reinterpret_cast<uint4*>(base + to[u]) = x[u];
      __syncwarp();
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  if (threadIdx.x == 0) *a.ticket = 0;
  for (int s = threadIdx.x >> 5; s < a.n_seqs; s += 8) {
    const CommitSeq q = commit_seq(a, s);
    if (lane == 0) a.lens_out[s] = q.n < 0 ? q.len : q.past + q.n;
  }
}

}  // namespace rpo
