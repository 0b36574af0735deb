// Pages of a caller-owned cache under reference counts: sequences that become the first tokens of others (fork), take or give
// back pages (reserve), and keep the accepted nodes of a tree of drafted tokens (commit).
//
// Bound by latency where little is copied (a few dependent look-ups and barriers), by HBM where much is (the copied rows
// once each way).  Fork and reserve change tables, counts and the stack of free pages in one cluster, whose barriers order the
// phases, and leave a list of pages to copy; a second kernel copies those in all layers, a CTA per page and group of planes (a
// plane is K or V of one KV head of one layer) with eight 16-byte pieces per thread in flight.  128 forks of 28 layers of 4 heads of
// 128: 41 to 45 us, half of it tables and counts.  Which page goes where is a matter of the order of forks or sequences alone, never of timing:
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

struct PageWs { PageCopy* copies; int *counts, *ticket; };      // [PG_MAX_ITEMS], [PG_MAX_ITEMS], two (the first zero between calls)

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

struct PageShared { int scan[PG_WARPS]; int first[PG_MAX_ITEMS + 1], taken; };   // first: pages needed, then released, before item i

__device__ __forceinline__ int warp_before(int v, int lane) {                 // sum of the lower lanes' values
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int n = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += n; }
  return incl - v;
}

// sh.first[i] = sum of count(i') over i' < i, for i <= n; all threads of the CTA.
template <typename F>
__device__ __forceinline__ void page_prefix(int n, PageShared& sh, F count) {
  static_assert(PG_WARPS == 32, "a warp scans the warps' sums");
  const int per = (n + PG_THREADS - 1) / PG_THREADS, i0 = threadIdx.x * per, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int c[PG_PER_THREAD], sum = 0;
#pragma unroll
  for (int k = 0; k < PG_PER_THREAD; ++k) {
    c[k] = k < per && i0 + k < n ? count(i0 + k) : 0;
    sum += c[k];
  }
  int before = warp_before(sum, lane);
  if (lane == 31) sh.scan[warp] = before + sum;
  __syncthreads();
  const int w = sh.scan[lane];
  before += (int)__reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
#pragma unroll
  for (int k = 0; k < PG_PER_THREAD; ++k) {
    if (k < per && i0 + k < n) sh.first[i0 + k] = before;
    before += c[k];
  }
  if (threadIdx.x == PG_THREADS - 1) sh.first[n] = before;
  __syncthreads();
}

// Items are served in order as long as the free pages last; those that need none always are.
__device__ __forceinline__ bool page_served(const PagePoolArgs& p, const PageShared& sh, int i, int n_free) {
  if (sh.first[i + 1] <= n_free || sh.first[i + 1] == sh.first[i]) return true;
  atomicOr(p.status, STATUS_NO_PAGES);
  return false;
}
__device__ __forceinline__ int page_taken(PageShared& sh, int n, int n_free) {          // pages that the served ones take
  if (sh.first[n] <= n_free) return sh.first[n];
  __syncthreads();
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

// f(slot, page) for the slots [lo, hi) of a table row, 32 PG_ROWS at a time: slot and page of each of a lane's PG_ROWS; page -1: no
// slot, or none of the pool.  Entries of slots below `marked` may carry PG_MARK; elsewhere a number with that bit is none of the pool.
constexpr int PG_ROWS = 4;

template <typename F>
__device__ __forceinline__ void page_slots(const PagePoolArgs& p, int s, int lo, int hi, F f, int marked = 0) {
  const int lane = threadIdx.x & 31;
  int32_t* row = p.table + (int64_t)s * p.stride;
  for (int j = lo; j < hi; j += 32 * PG_ROWS) {
    int slot[PG_ROWS], page[PG_ROWS];
#pragma unroll
    for (int k = 0; k < PG_ROWS; ++k) { slot[k] = j + 32 * k + lane; page[k] = slot[k] < hi ? row[slot[k]] : 0; }
#pragma unroll
    for (int k = 0; k < PG_ROWS; ++k) if (slot[k] >= hi || !p.in_pool(slot[k] < marked ? page[k] & ~PG_MARK : page[k])) page[k] = -1;
    f(slot, page);
  }
}

// The releasing half of a call.  dropped(i, f) calls f(slot, page) (as page_slots) for the pages that item i gives up, a warp
// together; finish(i) runs last, when the item's old table row is not needed any more.
//
// A page that this item alone holds is claimed at once: its count becomes PG_CLAIM plus the item's place, or, where a warp has one
// item of at most 1024 pages, 0, and a bit of the lane's remembers it (random 4-byte accesses of a few SMs are what this costs: 256
// sequences of 240 pages on average taken and given back 72 us with marks, 60 us with bits).  Other counts fall once all have been
// looked at (a count that is 1 because another item has given the page up is not this item's alone); where several items of one call
// give up the last references to a page, which is rare, two more passes find the first of them.
template <typename D, typename F>
__device__ __forceinline__ void page_release(const PagePoolArgs& p, int n, int n_free, int n_taken, PageShared& sh, D dropped, F finish) {
  const int lane = threadIdx.x & 31, warp = blockIdx.x * PG_WARPS + (threadIdx.x >> 5), warps = gridDim.x * PG_WARPS;
  auto place = [&](int i, int slot) { return PG_CLAIM + i * p.stride + slot; };
  volatile int* found = p.ws.ticket + 1;                 // 1: shared pages are given up; 2: one of them by all who held it
  const bool bits = n <= warps && p.stride <= 32 / PG_ROWS * 32 * PG_ROWS;
  uint32_t sole = 0;                                     // with bits: PG_ROWS for every call of f
  bool shared = false;
  if (blockIdx.x == 0 && threadIdx.x == 0) *found = 0;
  fa::cluster_sync();                                    // counts grow before they fall
  auto claimed = [&](int i, int slot, int page) { return page >= 0 && p.count_of(page) == place(i, slot); };
  for (int i = warp; i < n; i += warps) {
    int c = 0, call = 0;
    dropped(i, [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
      int r[PG_ROWS];
#pragma unroll
      for (int k = 0; k < PG_ROWS; ++k) r[k] = page[k] >= 0 ? p.count_of(page[k]) : 0;
#pragma unroll
      for (int k = 0; k < PG_ROWS; ++k) {
        if (page[k] < 0) continue;
        if (r[k] == 1) {
          p.refs[page[k]] = bits ? 0 : place(i, slot[k]);
          if (bits) sole |= 1u << (call * PG_ROWS + k);
          ++c;
        } else shared = true;
      }
      ++call;
    });
    c = (int)__reduce_add_sync(0xffffffffu, c);
    if (lane == 0) p.ws.counts[i] = c;
  }
  shared = __any_sync(0xffffffffu, shared);
  if (shared && lane == 0) *found = 1;
  fa::cluster_sync();
  bool again = false;
  if (*found) {
    if (shared)
      for (int i = warp; i < n; i += warps) {
        int call = 0;
        dropped(i, [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
#pragma unroll
          for (int k = 0; k < PG_ROWS; ++k)
            if (page[k] >= 0 && !(bits ? (sole >> (call * PG_ROWS + k)) & 1 : claimed(i, slot[k], page[k])) && atomicSub(p.refs + page[k], 1) == 1) *found = 2;
          ++call;
        });
      }
    fa::cluster_sync();
    again = *found == 2;
  }
  if (again) {
    for (int i = warp; i < n; i += warps)
      dropped(i, [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
#pragma unroll
        for (int k = 0; k < PG_ROWS; ++k) {
          if (page[k] < 0) continue;
          const int r = p.count_of(page[k]);
          if (r == 0 || r < PG_CLAIM / 2) atomicMin(p.refs + page[k], place(i, slot[k]));
        }
      });
    fa::cluster_sync();
    for (int i = warp; i < n; i += warps) {
      int c = 0;
      dropped(i, [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
#pragma unroll
        for (int k = 0; k < PG_ROWS; ++k) c += claimed(i, slot[k], page[k]);
      });
      c = (int)__reduce_add_sync(0xffffffffu, c);
      if (lane == 0) p.ws.counts[i] = c;
    }
    fa::cluster_sync();
  }
  page_prefix(n, sh, [&](int i) { return *(volatile int*)(p.ws.counts + i); });
  const int base = n_free - n_taken;
  for (int i = warp; i < n; i += warps) {
    int at = base + sh.first[i], call = 0;
    if (sh.first[i + 1] > sh.first[i])
      dropped(i, [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
        bool mine[PG_ROWS];
#pragma unroll
        for (int k = 0; k < PG_ROWS; ++k) mine[k] = bits && !again ? (sole >> (call * PG_ROWS + k)) & 1 : claimed(i, slot[k], page[k]);
        ++call;
#pragma unroll
        for (int k = 0; k < PG_ROWS; ++k) {
          const unsigned who = __ballot_sync(0xffffffffu, mine[k]);
          const int to = at + __popc(who & ((1u << lane) - 1));
          if (mine[k]) {
            if (!bits || again) p.refs[page[k]] = 0;
            if (to < p.n_blocks) p.free[to] = page[k]; else p.bad_length();
          }
          at += __popc(who);
        }
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
  // what a warp's first fork is stays in registers: behind a cluster barrier each look is one to L2 again
  struct Fork { int src, dst, len, held, copy; };
  Fork mine = {0, 0, 0, 0, -1};
  auto fork = [&](int i) {
    if (i == warp) return mine;
    return Fork{a.src[i], a.dst[i], a.lens[i], p.pages_held(a.dst[i]), p.ws.copies[i].to};
  };
  for (int i = warp, k = 0; i < a.n; i += warps, ++k) {
    PageCopy copy = {-1, -1, 0, 0};
    if (valid(i) && page_served(p, sh, i, n_free)) {
      ok.set(k);
      const int len = a.lens[i], whole = len / KV_BLOCK, s = a.src[i];
      if (k == 0) mine = Fork{s, a.dst[i], len, p.pages_held(a.dst[i]), -1};
      page_slots(p, s, 0, whole, [&](const int (&)[PG_ROWS], const int (&page)[PG_ROWS]) {
#pragma unroll
        for (int k = 0; k < PG_ROWS; ++k) if (page[k] >= 0) atomicAdd(p.refs + page[k], 1);
      });
      if (len % KV_BLOCK) {
        copy.from = p.table[(int64_t)s * p.stride + whole];
        copy.to = p.free[n_free - 1 - sh.first[i]];
        if (!p.in_pool(copy.to)) copy.to = -1;
        if (p.in_pool(copy.from) && copy.to >= 0) copy.rows = len % KV_BLOCK;
        if (lane == 0 && copy.to >= 0) p.refs[copy.to] = 1;
      }
    }
    if (k == 0) mine.copy = copy.to;
    if (lane == 0) p.ws.copies[i] = copy;
  }
  page_release(p, a.n, n_free, n_taken, sh,
               [&](int i, auto f) {
                 if (!ok.get((i - warp) / warps)) return;
                 const Fork x = fork(i);
                 page_slots(p, x.dst, 0, x.held, f);
               },
               [&](int i) {
                 if (!ok.get((i - warp) / warps)) return;
                 const Fork x = fork(i);
                 const int whole = x.len / KV_BLOCK, part = x.len % KV_BLOCK ? 1 : 0;
                 const int32_t* from = p.table + (int64_t)x.src * p.stride;
                 int32_t* to = p.table + (int64_t)x.dst * p.stride;
#pragma unroll 4
                 for (int j = lane; j < whole; j += 32) to[j] = from[j];
                 if (lane == 0) {
                   if (part) to[whole] = x.copy;
                   p.held[x.dst] = whole + part;
                   if (a.lens_out) a.lens_out[x.dst] = x.len;
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
  auto look = [&](int s) {
    ReserveSeq x;
    x.held = p.pages_held(s);
    const int target = p.clamped(a.target[s], most);
    x.len = p.clamped(min(p.clamped(a.lens[s], most), target), x.held * KV_BLOCK);
    x.want = (target + KV_BLOCK - 1) / KV_BLOCK;
    return x;
  };
  // a warp's first sequence stays in registers: behind a cluster barrier each look is one to L2 again
  const ReserveSeq mine = warp < n ? look(warp) : ReserveSeq{0, 0, 0};
  auto seq = [&](int s) { return s == warp ? mine : look(s); };
  for (int s = warp; s < n; s += warps) {
    const ReserveSeq x = seq(s);
    int32_t* row = p.table + (int64_t)s * p.stride;
    int need = max(0, x.want - x.held);
    int replaced = 0;
    page_slots(p, s, x.len / KV_BLOCK, min(x.held, x.want), [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
      int r[PG_ROWS];
#pragma unroll
      for (int k = 0; k < PG_ROWS; ++k) r[k] = page[k] >= 0 ? p.count_of(page[k]) : 0;
#pragma unroll
      for (int k = 0; k < PG_ROWS; ++k) {
        if (r[k] > 1) { row[slot[k]] = page[k] | PG_MARK; ++replaced; }
        else if (page[k] < 0 && slot[k] < min(x.held, x.want) && row[slot[k]] >= 0) row[slot[k]] = -1;      // (a number that could pass for a mark)
      }
    });
    need += (int)__reduce_add_sync(0xffffffffu, replaced);
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
                 page_slots(p, s, x.len / KV_BLOCK, x.held, [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
                   int old[PG_ROWS];
#pragma unroll
                   for (int k = 0; k < PG_ROWS; ++k) {
                     old[k] = -1;
                     if (page[k] >= 0 && (page[k] & PG_MARK)) {        // (below want alone)
                       old[k] = p.count_of(page[k] & ~PG_MARK) - PG_OLD;
                       if (old[k] < 0 || old[k] >= p.n_blocks) old[k] = -1;
                     } else if (slot[k] >= x.want) old[k] = page[k];
                   }
                   f(slot, old);
                 }, x.want);
               },
               [&](int s) {
                 if (!ok.get((s - warp) / warps)) return;
                 const ReserveSeq x = seq(s);
                 page_slots(p, s, x.len / KV_BLOCK, min(x.held, x.want), [&](const int (&slot)[PG_ROWS], const int (&page)[PG_ROWS]) {
#pragma unroll
                   for (int k = 0; k < PG_ROWS; ++k) {
                     if (page[k] < 0 || !(page[k] & PG_MARK)) continue;
                     p.table[(int64_t)s * p.stride + slot[k]] = page[k] & ~PG_MARK;
                     p.refs[page[k] & ~PG_MARK] = 1;
                   }
                 }, x.want);
                 __syncwarp();
                 if (lane == 0) p.held[s] = x.want;
               });
}

// The first rows of pages, in every plane: a CTA takes one page and `per` planes, every thread the same 16 bytes of several planes.
constexpr int PG_LOADS = 8, PG_MOVE_THREADS = 256, PG_PLANES = 64;

__global__ void __launch_bounds__(PG_MOVE_THREADS, 4) copy_pages_kernel(const __grid_constant__ PageLayers l, const PageCopy* copies, int n, int per, bool rare) {
  __shared__ uint8_t* s_plane[PG_PLANES];                // `per` is at most that
  if (rare) {                                            // as a rule there is nothing to copy: one look instead of one per page
    bool any = false;
    for (int i = threadIdx.x; i < n; i += PG_MOVE_THREADS) any = any || copies[i].rows != 0;
    if (!__syncthreads_or(any)) return;
  }
  const int parts = (l.planes() + per - 1) / per;
  for (int64_t w = blockIdx.x; w < (int64_t)n * parts; w += gridDim.x) {
    const PageCopy c = copies[w / parts];
    const int pieces = c.rows * l.row_bytes / 16, p0 = (int)(w % parts) * per, planes = min(l.planes() - p0, per);
    if (pieces == 0) continue;
    const int64_t page_bytes = (int64_t)KV_BLOCK * l.row_bytes, from = c.from * page_bytes, to = c.to * page_bytes;
    __syncthreads();                                     // the last planes are read
    for (int p = threadIdx.x; p < planes; p += PG_MOVE_THREADS) s_plane[p] = l.plane(p0 + p);
    __syncthreads();
    const int together = max(1, PG_MOVE_THREADS / pieces), sub = pieces <= PG_MOVE_THREADS ? threadIdx.x / pieces : 0;      // planes side by side
    if (sub >= together) continue;
    for (int i = pieces <= PG_MOVE_THREADS ? threadIdx.x - sub * pieces : threadIdx.x; i < pieces; i += PG_MOVE_THREADS)
      for (int p = sub; p < planes; p += together * PG_LOADS) {
        uint4 x[PG_LOADS];
#pragma unroll
        for (int u = 0; u < PG_LOADS; ++u) if (p + u * together < planes) x[u] = reinterpret_cast<const uint4*>(s_plane[p + u * together] + from)[i];
#pragma unroll
        for (int u = 0; u < PG_LOADS; ++u) if (p + u * together < planes) reinterpret_cast<uint4*>(s_plane[p + u * together] + to)[i] = x[u];
      }
  }
}

// Commit: the rows of the accepted nodes, in ascending order, to the front of the tree's slots.  A CTA takes a sequence and `per`
// planes: it looks the rows' places up once, then moves the rows in order, PG_LOADS pieces per thread at once, all of them read before
// any is written; a row's source never lies before its destination, so what is read later has not been overwritten.  The CTA that ends
// last writes the lengths, which the others have read.
constexpr int PG_MOVES = 256;                             // rows whose places are kept at once

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

__global__ void __launch_bounds__(PG_MOVE_THREADS, 4) commit_path_kernel(const __grid_constant__ PageLayers l, CommitArgs a, int per) {
  __shared__ int s_last;
  __shared__ int2 s_move[PG_MOVES];                      // rows inside a plane, from and to; to -1: stays
  __shared__ uint8_t* s_plane[PG_PLANES];                // `per` is at most that
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lanes = l.row_bytes / 16;      // 16-byte pieces of a row
  const int parts = (l.planes() + per - 1) / per;
  for (int64_t w = blockIdx.x; w < (int64_t)a.n_seqs * parts; w += gridDim.x) {
    const int s = (int)(w / parts), p0 = (int)(w % parts) * per, p1 = min(l.planes(), p0 + per);
    const CommitSeq q = commit_seq(a, s);
    const int32_t* path = a.path + (int64_t)s * a.path_stride;
    const int32_t* row = a.table + (int64_t)s * a.stride;
    auto place = [&](int slot) {
      const int page = row[slot / KV_BLOCK];
      if (page < 0 || page >= l.n_blocks) { atomicOr(a.status, STATUS_BAD_BLOCK); return -1; }
      return page * KV_BLOCK + slot % KV_BLOCK;
    };
    for (int first = 0; first < q.n; first += PG_MOVES) {
      const int n = min(PG_MOVES, q.n - first);
      __syncthreads();                                   // the last rows' places are read
      for (int p = p0 + threadIdx.x; p < p1; p += PG_MOVE_THREADS) s_plane[p - p0] = l.plane(p);
      for (int i = threadIdx.x; i < n; i += PG_MOVE_THREADS) {
        const int node = path[first + i];
        int2 m = make_int2(0, -1);
        if (node != first + i) { m.x = place(q.past + node); m.y = place(q.past + first + i); if (m.x < 0) m.y = -1; }
        s_move[i] = m;
      }
      __syncthreads();
      // as many rows, and planes, as PG_LOADS pieces of every thread hold: all are read before any is written
      const int rows = min(n, PG_LOADS * PG_MOVE_THREADS / lanes);
      for (int r0 = 0; r0 < n; r0 += rows) {
        const int nr = min(rows, n - r0), together = PG_LOADS * PG_MOVE_THREADS / (lanes * nr);
        const int first_q = threadIdx.x / lanes / nr, first_r = threadIdx.x / lanes % nr, step_q = PG_MOVE_THREADS / lanes / nr, step_r = PG_MOVE_THREADS / lanes % nr;
        for (int p = p0; p < p1; p += together) {
          const int planes = min(together, p1 - p);
          uint4 x[PG_LOADS];
          // this thread's pieces: planes q, rows r of them
          auto pieces = [&](auto f) {
            int q = first_q, r = first_r;
#pragma unroll
            for (int u = 0; u < PG_LOADS; ++u) {
              if (q < planes) {
                const int2 m = s_move[r0 + r];
                if (m.y >= 0) f(u, s_plane[p - p0 + q] + threadIdx.x % lanes * 16, m);
              }
              q += step_q; r += step_r;
              if (r >= nr) { r -= nr; ++q; }
            }
          };
          pieces([&](int u, uint8_t* base, const int2& m) { x[u] = *reinterpret_cast<const uint4*>(base + (int64_t)m.x * l.row_bytes); });
          __syncthreads();
          pieces([&](int u, uint8_t* base, const int2& m) { *reinterpret_cast<uint4*>(base + (int64_t)m.y * l.row_bytes) = x[u]; });
        }
      }
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
  for (int s = warp; s < a.n_seqs; s += PG_MOVE_THREADS / 32) {
    const CommitSeq q = commit_seq(a, s);
    if (lane == 0) a.lens_out[s] = q.n < 0 ? q.len : q.past + q.n;
  }
}

}  // namespace rpo
