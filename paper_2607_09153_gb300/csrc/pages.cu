// The pages' bookkeeping between two steps of a search: kvprm_cache_fork (sequences dropped, doubled and given room) and
// kvprm_cache_compact (pages in use moved to the pool's beginning).
//
// Either is two launches.  The first works out references and who is copied where: one cluster of CTAs, whose barrier
// separates the steps, because each step needs what all threads found in the one before and the whole is a few thousand to a few
// hundred thousand numbers.  The second writes the tables and copies pages, warp by warp in pieces of 4 KB, over all layers of all
// pools; it is launched beside the first one's end and learns there how many there are.  (Few of both are the cluster's too.)
// Nothing is decided by who comes first: counts are sums, of several that want a page the lowest sequence has it, free pages go
// by their numbers.
//
// What bounds them, measured on a GB300: memory, once copies are many (462 pages of 0.46 MB compacted in 77 us, 67 of them the
// copies', 6,400 GB/s; 217 pages of 0.92 MB copied in a fork of 64 sequences into 256 in 55 us, 44 of them 199 MB written from
// pages that L2 keeps); the steps' latencies before that, 7 to 10 us of a fork and 5 of a compaction (three cluster barriers each, each
// behind loads or atomics of the step, and a fourth where the cluster writes tables and copies itself).
#include <cuda_runtime.h>

#include <algorithm>
#include <utility>

#include "ptx.cuh"
#include "rope.h"

namespace kvprm {

namespace {

constexpr int kThreads = 1024, kCluster = 8;
constexpr int kCopyCtas = 4;       // of an SM
constexpr int kMost = 1 << 24;     // pages of a block table
constexpr int kSmall = 1024;       // pieces, or segments of tables, that the cluster alone sees to
constexpr int kPage = 16, kNobody = 0x7FFFFFFF;
constexpr int kCopyThreads = 256, kCopyUnroll = 8, kPiece = 32 * 16 * kCopyUnroll;   // of a warp: 4 KB

// ---------------------------------------------------------------- a cluster's steps
__device__ __forceinline__ int cluster_thread() { return static_cast<int>(cluster_rank()) * kThreads + threadIdx.x; }
constexpr int kAll = kCluster * kThreads;
static_assert(kAll == KVPRM_MAX_SEQS, "a thread for each new sequence");

// All threads of the cluster meet, and see what any of them has written.
__device__ __forceinline__ void step() {
  __syncwarp();
  cluster_sync();
}

// What the CTAs of the cluster told each other: each writes its number to all, and after the cluster's barrier each
// has all of them.
__device__ __forceinline__ void tell(uint64_t* told, uint64_t value) {   // told[kCluster], one thread
  const uint32_t me = cluster_rank();
  for (uint32_t r = 0; r < kCluster; ++r) {
    const uint32_t to = cluster_addr(told + me, r);
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(value) : "memory");
  }
}

// The sum over the CTA's threads before this one; *total over all.
__device__ __forceinline__ uint64_t cta_before(uint64_t v, uint64_t* s_warp, uint64_t* total) {
  const int lane = threadIdx.x & 31;
  uint64_t scan = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint64_t up = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += up;
  }
  __syncthreads();   // (the last use's sums have been read)
  if (lane == 31) s_warp[threadIdx.x >> 5] = scan;
  __syncthreads();
  uint64_t sum = s_warp[lane];   // one of each of the 32 warps
  const uint64_t own = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint64_t up = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += up;
  }
  const int warp = threadIdx.x >> 5;
  *total = __shfl_sync(0xffffffffu, sum, 31);
  return __shfl_sync(0xffffffffu, sum - own, warp) + scan - v;
}

// Indices 0 .. n - 1 are shared out as one range a CTA.
struct Range {
  int lo, hi;
  __device__ __forceinline__ explicit Range(int n) {
    const int per = (n + kCluster - 1) / kCluster;
    lo = min(n, per * static_cast<int>(cluster_rank()));
    hi = min(n, lo + per);
  }
  __device__ __forceinline__ int mine() const { return lo + threadIdx.x < hi ? lo + static_cast<int>(threadIdx.x) : -1; }
};
__device__ __forceinline__ uint64_t told_before(const uint64_t* told) {
  uint64_t sum = 0;
  for (uint32_t i = 0; i < cluster_rank(); ++i) sum += told[i];
  return sum;
}
__device__ __forceinline__ uint64_t sum_told(const uint64_t* told) {
  uint64_t sum = 0;
  for (int i = 0; i < kCluster; ++i) sum += told[i];
  return sum;
}

// Calls f(row, begin, end, lane) for each row of a table in segments of 128 entries (2^30 at most), for warp `warp` of `warps`.
constexpr int kSegment = 128;
static_assert(int64_t{KVPRM_MAX_SEQS} * (kMost / kSegment) <= 1 << 30, "segments");
template <typename F>
__device__ __forceinline__ void each_segment(int rows, int width, uint32_t warp, uint32_t warps, F f) {
  const uint32_t per_row = (width + kSegment - 1) / kSegment, lane = threadIdx.x & 31;
  for (uint32_t i = warp; i < rows * per_row; i += warps) {
    const uint32_t row = i / per_row;
    const int begin = static_cast<int>(i - row * per_row) * kSegment;
    f(static_cast<int>(row), begin, min(width, begin + kSegment), static_cast<int>(lane));
  }
}
constexpr uint32_t kOnce = 1u << 31;   // `warps` for a warp's first segment alone

// ---------------------------------------------------------------- fork
// A new sequence's row, as the last step writes it: its parent (-1: none), pages taken over, pages in all, its place among the
// free pages (kCopied: the first of them is its last page's copy).
constexpr int32_t kCopied = 1 << 30;
struct ForkLaunch {
  kvprm_fork f;
  int32_t *first, *free_pages, *count;   // scratch; first: who is the first of the new sequences to end inside a page;
                                         // count: copies, and pages that are free before any is given away
  int4* rows;
  int2* pairs;
};

// A sequence before the fork: pages that it holds, and full ones (none where its length cannot be).
struct Held {
  int32_t len, pages, full;
  __device__ __forceinline__ Held(const kvprm_fork& f, int s) {
    len = __ldg(f.lens + s);
    const bool bad = len < 0 || static_cast<int64_t>(len) > static_cast<int64_t>(kPage) * f.max_blocks;
    pages = bad ? 0 : (len + kPage - 1) / kPage;
    full = bad ? 0 : len / kPage;
  }
};

// What a new sequence takes over and wants.
struct Heir {
  int32_t parent = -1, len = 0, pages = 0, last = -1, end = 0;   // last: the page that it ends inside; end: pages that it is to have
  int64_t lacking = 0;                                           // pages beyond its table's width
  __device__ __forceinline__ Heir(const kvprm_fork& f, int i) {
    if (i < 0) return;
    parent = __ldg(f.parents + i);
    const int64_t room = f.room ? max(0, __ldg(f.room + i)) : 0;
    if (parent < 0 || parent >= f.n_seqs) parent = -1;
    bool bad = false;
    if (parent >= 0) {
      const Held h(f, parent);
      len = h.len;
      bad = h.pages == 0 && h.len != 0;
      pages = min(h.pages, f.width);
      if (h.full < pages) {
        last = __ldg(f.block_table + static_cast<int64_t>(parent) * f.max_blocks + h.full);
        if (last < 0 || last >= f.n_pages) last = -1;
      }
    }
    const int64_t want = bad ? 0 : (len + room + kPage - 1) / kPage;
    end = max(static_cast<int32_t>(min(want, static_cast<int64_t>(f.width))), pages);
    lacking = max(int64_t{0}, want - end);
  }
};

// Everything but the tables and the copies.
__device__ __forceinline__ void plan(const ForkLaunch& a) {
  __shared__ uint64_t s_warp[32], s_need[kCluster], s_free[kCluster], s_lacking[kCluster];
  __shared__ int32_t s_heirs[KVPRM_MAX_SEQS];   // of each sequence: every CTA counts all
  const kvprm_fork& f = a.f;
  const int me = cluster_thread();
  const int n_pages = static_cast<int>(f.n_pages);
  // (what hangs on nothing is loaded first)
  const int i = Range(f.n_new).mine();   // this thread's new sequence (there are no more of them than threads)
  const int32_t refs0 = me < n_pages ? __ldg(f.refs + me) : 0, parent0 = static_cast<int>(threadIdx.x) < f.n_new ? __ldg(f.parents + threadIdx.x) : -1;
  for (int s = threadIdx.x; s < f.n_seqs; s += kThreads) s_heirs[s] = 0;
  const Heir h(f, i);
  __syncthreads();
  if (parent0 >= 0 && parent0 < f.n_seqs) atomicAdd(s_heirs + parent0, 1);
  for (int j = threadIdx.x + kThreads; j < f.n_new; j += kThreads) {
    const int parent = __ldg(f.parents + j);
    if (parent >= 0 && parent < f.n_seqs) atomicAdd(s_heirs + parent, 1);
  }
  for (int p = me; p < n_pages; p += kAll) {
    f.refs_out[p] = p == me ? refs0 : __ldg(f.refs + p);
    a.first[p] = kNobody;
  }
  // (the warp's first segment of the old tables is on its way over the barrier)
  const uint32_t warp = (threadIdx.x >> 5) * kCluster + cluster_rank();
  constexpr int kFirst = kSegment / 32;
  int32_t ahead[kFirst];
  each_segment(f.n_seqs, f.max_blocks, warp, kOnce, [&](int s, int begin, int end, int lane) {
    const int stop = min(end, Held(f, s).pages);
#pragma unroll
    for (int x = 0; x < kFirst; ++x) {
      const int b = begin + lane + 32 * x;
      ahead[x] = b < stop ? __ldg(f.block_table + static_cast<int64_t>(s) * f.max_blocks + b) : -1;
    }
  });
  step();

  // full pages: one reference less, and one more for each that continues the sequence; of those that end inside a page the first
  if (h.last >= 0) atomicMin(a.first + h.last, i);
  bool first = true;
  auto change = [&](const Held& held, int heirs, int b, int32_t page) {
    const int by = (b < held.full && b < f.width ? heirs : 0) - 1;
    if (page >= 0 && page < n_pages && by != 0) atomicAdd(f.refs_out + page, by);
  };
  each_segment(f.n_seqs, f.max_blocks, warp, kAll / 32, [&](int s, int begin, int end, int lane) {
    const Held held(f, s);
    const int heirs = s_heirs[s];
    if (first) {
      first = false;
#pragma unroll
      for (int x = 0; x < kFirst; ++x) change(held, heirs, begin + lane + 32 * x, ahead[x]);
      return;
    }
    const int32_t* row = f.block_table + static_cast<int64_t>(s) * f.max_blocks;
    const int stop = min(end, held.pages);
#pragma unroll 4
    for (int b = begin + lane; b < stop; b += 32) change(held, heirs, b, __ldg(row + b));
  });
  step();

  // A page that ends inside is kept by the first who ends in it if nobody else holds it, and copied for the others; what
  // nobody holds or ends in is free.
  const bool copied = h.last >= 0 && !(__ldcg(f.refs_out + h.last) <= 0 && __ldcg(a.first + h.last) == i);
  auto is_free = [&](int p) { return p >= 0 && __ldcg(f.refs_out + p) <= 0 && __ldcg(a.first + p) == kNobody; };
  const Range pages(n_pages);
  const int p0 = pages.mine();
  const bool free0 = is_free(p0);
  // of a CTA's first 1,024 pages and its new sequences at once: free pages (11 bits), copies (11), pages wanted (31)
  const uint64_t v = (static_cast<uint64_t>(free0) << 52) | (static_cast<uint64_t>(copied) << 40) |
                     static_cast<uint64_t>(static_cast<uint32_t>(h.end - h.pages) + (copied ? 1u : 0u));
  uint64_t total;
  const uint64_t before = cta_before(v, s_warp, &total);
  uint64_t frees = total >> 52;
  for (int q = pages.lo + kThreads; q < pages.hi; q += kThreads) {
    const int p = q + static_cast<int>(threadIdx.x);
    frees += __syncthreads_count(is_free(p < pages.hi ? p : -1));
  }
  uint64_t lacking = 0;
  if (__syncthreads_or(h.lacking > 0)) cta_before(h.lacking, s_warp, &lacking);
  if (threadIdx.x == 0) {
    tell(s_need, total & ((uint64_t{1} << 52) - 1));
    tell(s_free, frees);
    tell(s_lacking, lacking);
  }
  step();

  const uint64_t needed = sum_told(s_need), mask = (uint64_t{1} << 40) - 1;
  const int64_t wanted = static_cast<int64_t>(needed & mask), have = static_cast<int64_t>(sum_told(s_free));
  if (i >= 0) {
    const uint64_t at = told_before(s_need) + (before & ((uint64_t{1} << 52) - 1));
    const int32_t place = static_cast<int32_t>(at & mask);
    a.rows[i] = make_int4(h.parent, h.pages, h.end, place | (copied ? kCopied : 0));
    if (copied) a.pairs[at >> 40] = make_int2(h.last, place);
    if (h.last >= 0 && !copied) f.refs_out[h.last] = 1;         // kept
    f.lens_out[i] = h.len;
  }
  auto give = [&](int p, int64_t rank) {
    if (rank >= wanted) return;
    a.free_pages[rank] = p;
    f.refs_out[p] = 1;
  };
  int64_t rank = static_cast<int64_t>(told_before(s_free));
  if (free0) give(p0, rank + static_cast<int64_t>(before >> 52));
  rank += static_cast<int64_t>(total >> 52);
  for (int q = pages.lo + kThreads; q < pages.hi; q += kThreads) {
    const int p = q + static_cast<int>(threadIdx.x) < pages.hi ? q + static_cast<int>(threadIdx.x) : -1;
    const bool free = is_free(p);
    const int64_t at = rank + static_cast<int64_t>(cta_before(free ? 1 : 0, s_warp, &total));
    if (free) give(p, at);
    rank += static_cast<int64_t>(total);
  }
  if (me == 0) {
    f.counts[0] = static_cast<int32_t>(max(int64_t{0}, have - wanted));
    f.counts[1] = static_cast<int32_t>(min(int64_t{kNobody}, max(int64_t{0}, wanted - have) + static_cast<int64_t>(sum_told(s_lacking))));
    a.count[0] = static_cast<int>(needed >> 40);
    a.count[1] = static_cast<int>(have);
  }
}

// A new sequence's pages: those that it takes over, and its own.
__device__ __forceinline__ void fork_tables(const ForkLaunch& a, uint32_t warp, uint32_t warps) {
  const kvprm_fork& f = a.f;
  const int32_t have = __ldcg(a.count + 1);
  each_segment(f.n_new, f.width, warp, warps, [&](int r, int begin, int end, int lane) {
    const int4 row = __ldcg(a.rows + r);
    const int32_t first = row.w & (kCopied - 1), mine = row.y - (row.w & kCopied ? 1 : 0);
    const int32_t* from = f.block_table + static_cast<int64_t>(max(row.x, 0)) * f.max_blocks;
    int32_t* out = f.table_out + static_cast<int64_t>(r) * f.width;
#pragma unroll 4
    for (int b = begin + lane; b < end; b += 32) {
      const int32_t k = first + b - mine;
      out[b] = b < mine ? __ldg(from + b) : b < row.z && k < have ? __ldcg(a.free_pages + k) : -1;
    }
  });
}
// Where a copy goes: its place among the free pages; -1: there is none.
__device__ __forceinline__ int32_t copy_to(const ForkLaunch& a, int32_t place) {
  return place < __ldcg(a.count + 1) ? __ldcg(a.free_pages + place) : -1;
}

// ---------------------------------------------------------------- compact
struct CompactLaunch {
  kvprm_compact f;
  int32_t *low, *high, *count;   // scratch: free pages before the first `live`, and pages in use by how many are before them
  int2* pairs;
};

__device__ __forceinline__ void plan(const CompactLaunch& a) {
  __shared__ uint64_t s_warp[32], s_live[kCluster], s_below;
  const kvprm_compact& f = a.f;
  cluster_arrive();   // (the CTAs tell each other something only when all have begun)
  const int me = cluster_thread(), n_pages = static_cast<int>(f.n_pages);
  const Range pages(n_pages);
  const int p0 = pages.mine(), refs0 = p0 < 0 ? 0 : __ldg(f.refs + p0);
  uint64_t total;
  const uint64_t before = cta_before(refs0 > 0 ? 1 : 0, s_warp, &total);   // of the CTA's first 1,024 pages
  uint64_t used = total;
  for (int q = pages.lo + kThreads; q < pages.hi; q += kThreads) {
    const int p = q + static_cast<int>(threadIdx.x);
    used += __syncthreads_count(p < pages.hi && __ldg(f.refs + p) > 0);
  }
  __syncwarp();
  cluster_wait();
  if (threadIdx.x == 0) tell(s_live, used);
  step();
  const int live = static_cast<int>(sum_told(s_live));
  // of the first `live` pages, those in use: what is free among them are as many as are in use behind
  auto sort = [&](int p, int refs, int rank) {   // rank: pages in use before this one
    if (p == live)
      for (uint32_t r = 0; r < kCluster; ++r)
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_addr(&s_below, r)), "l"(static_cast<uint64_t>(rank)) : "memory");
    if (p < live && refs <= 0) a.low[p - rank] = p;
    if (p >= live && refs > 0) a.high[rank] = p;
    if (p < live && refs > 0) f.refs_out[p] = refs;
    if (p >= live) f.refs_out[p] = 0;
    f.moved[p] = p < live && refs > 0 ? p : -1;
  };
  int rank = static_cast<int>(told_before(s_live));
  if (p0 >= 0) sort(p0, refs0, rank + static_cast<int>(before));
  rank += static_cast<int>(total);
  for (int q = pages.lo + kThreads; q < pages.hi; q += kThreads) {
    const int p = q + static_cast<int>(threadIdx.x), refs = p < pages.hi ? __ldg(f.refs + p) : 0;
    const uint64_t at = cta_before(refs > 0 ? 1 : 0, s_warp, &total);
    if (p < pages.hi) sort(p, refs, rank + static_cast<int>(at));
    rank += static_cast<int>(total);
  }
  step();
  const int below = live < n_pages ? static_cast<int>(s_below) : live, moves = live - below;
  for (int j = me; j < moves; j += kAll) {
    const int from = __ldcg(a.high + below + j), to = __ldcg(a.low + j);
    a.pairs[j] = make_int2(from, to);
    f.moved[from] = to;
    f.refs_out[to] = __ldg(f.refs + from);
  }
  if (me == 0) {
    *a.count = moves;
    f.counts[0] = live;
    f.counts[1] = moves;
  }
}

__device__ __forceinline__ void compact_tables(const CompactLaunch& a, uint32_t warp, uint32_t warps) {
  const kvprm_compact& f = a.f;
  const int n_pages = static_cast<int>(f.n_pages);
  each_segment(f.n_seqs, f.max_blocks, warp, warps, [&](int s, int begin, int end, int lane) {
    const int32_t len = __ldg(f.lens + s);
    const int64_t held = len < 0 || static_cast<int64_t>(len) > static_cast<int64_t>(kPage) * f.max_blocks ? 0 : (len + kPage - 1) / kPage;
    const int64_t row = static_cast<int64_t>(s) * f.max_blocks;
#pragma unroll 4
    for (int b = begin + lane; b < end; b += 32) {
      int32_t page = -1;
      if (b < held) {
        page = __ldg(f.block_table + row + b);
        if (page >= 0 && page < n_pages) page = __ldcg(f.moved + page);
      }
      f.table_out[row + b] = page;
    }
  });
}

// ---------------------------------------------------------------- copying
// N: room for pools; a launch with arguments of 4 KB takes the host two microseconds more than one with four pools.
template <int N>
struct CopyLaunch {
  kvprm_pool pool[N];
  int32_t first[N + 1];   // pieces of a page of the pools before
  int32_t n_pools;
};
constexpr int kFewPools = 4;

// T: ForkLaunch or CompactLaunch, whose tables are written first.
__device__ __forceinline__ void tables(const ForkLaunch& t, uint32_t warp, uint32_t warps) { fork_tables(t, warp, warps); }
__device__ __forceinline__ void tables(const CompactLaunch& t, uint32_t warp, uint32_t warps) { compact_tables(t, warp, warps); }
__device__ __forceinline__ int32_t copy_to(const CompactLaunch&, int32_t page) { return page; }

// A fork's copies come of few pages, which stay in L2 (217 copies of 64 sequences' pages, 199 MB: 46 us, and 58 with loads that
// leave L2 first); what a compaction moves is read once.
__device__ __forceinline__ uint4 load_piece(const ForkLaunch&, const uint8_t* p) { return __ldcg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ uint4 load_piece(const CompactLaunch&, const uint8_t* p) { return __ldcs(reinterpret_cast<const uint4*>(p)); }

// The copies, for warp `first` of `warps`.
template <int N, typename T>
__device__ __forceinline__ void copies(const CopyLaunch<N>& a, const T& t, int64_t first, int64_t warps) {
  const int lane = threadIdx.x & 31, per_copy = a.first[a.n_pools];
  const int64_t items = static_cast<int64_t>(__ldcg(t.count)) * per_copy;
  for (int64_t i = first; i < items; i += warps) {
    const int64_t j = i / per_copy;
    int r = static_cast<int>(i - j * per_copy), k = 0;
    while (r >= a.first[k + 1]) ++k;
    r -= a.first[k];
    const kvprm_pool& p = a.pool[k];
    const int pieces = static_cast<int>((p.page_bytes + kPiece - 1) / kPiece), layer = r / pieces, piece = r - layer * pieces;
    int2 pair = __ldcg(t.pairs + j);
    pair.y = copy_to(t, pair.y);
    uint8_t* base = static_cast<uint8_t*>(p.base) + layer * p.layer_stride + static_cast<int64_t>(piece) * kPiece + lane * 16;
    if (pair.y < 0) continue;   // no page was free
    const uint8_t* src = base + pair.x * p.page_stride;
    uint8_t* dst = base + pair.y * p.page_stride;
    const int64_t left = p.page_bytes - static_cast<int64_t>(piece) * kPiece - lane * 16;   // bytes from this lane's first on
    uint4 v[kCopyUnroll];
#pragma unroll
    for (int x = 0; x < kCopyUnroll; ++x)
      if (x * 512 < left) v[x] = load_piece(t, src + x * 512);
#pragma unroll
    for (int x = 0; x < kCopyUnroll; ++x)
      if (x * 512 < left) __stcs(reinterpret_cast<uint4*>(dst + x * 512), v[x]);
  }
}

template <typename T>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 1) plan_kernel(const __grid_constant__ T t) {
  grid_dep_launch();
  plan(t);
}
template <int N, typename T>
__global__ void __launch_bounds__(kCopyThreads, kCopyCtas) copy_kernel(const __grid_constant__ CopyLaunch<N> a, const __grid_constant__ T t) {
  const int warp = threadIdx.x >> 5;
  const uint32_t warps = gridDim.x * (kCopyThreads / 32);
  grid_dep_wait();
  tables(t, warp * gridDim.x + blockIdx.x, warps);
  copies(a, t, static_cast<int64_t>(blockIdx.x) * (kCopyThreads / 32) + warp, warps);
}
// All of a small call by the cluster alone.
template <typename T>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 1)
    small_kernel(const __grid_constant__ CopyLaunch<kFewPools> a, const __grid_constant__ T t) {
  plan(t);
  step();
  const uint32_t warp = (threadIdx.x >> 5) * kCluster + cluster_rank();
  tables(t, warp, kAll / 32);
  copies(a, t, warp, kAll / 32);
}

// ---------------------------------------------------------------- host
bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int64_t round_up(int64_t n) { return (n + 255) / 256 * 256; }

struct Part {   // an array of a call
  const void* p;
  int64_t bytes;
};
bool meet(const Part& a, const Part& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.bytes > 0 && b.bytes > 0 && x < y + b.bytes && y < x + a.bytes;
}

// Pages in memory: `layers` times `n` of `bytes`, with strides that are not negative (0 where there is one).
using Wide = __int128;   // (sums of strides of any size)
struct Box {
  Wide at, layer_stride, stride;
  int64_t layers, n, bytes;
  Box() {}
  explicit Box(const Part& a) : at(reinterpret_cast<uintptr_t>(a.p)), layer_stride(0), stride(0), layers(1), n(1), bytes(a.bytes) {}
  Box(const kvprm_pool& p, int64_t n_pages)
      : at(reinterpret_cast<uintptr_t>(p.base)), layer_stride(p.layers > 1 ? p.layer_stride : 0), stride(n_pages > 1 ? p.page_stride : 0),
        layers(p.layers), n(n_pages), bytes(p.page_bytes) {
    if (layer_stride < 0) at += layer_stride * (layers - 1), layer_stride = -layer_stride;
    if (stride < 0) at += stride * (n - 1), stride = -stride;
  }
  bool empty() const { return layers <= 0 || n <= 0 || bytes <= 0; }
  Wide row() const { return stride * (n - 1) + bytes; }   // from a layer's first page to its end
  Wide end() const { return at + layer_stride * (layers - 1) + row(); }
};
Wide floor_div(Wide a, Wide b) { return a / b - (a % b < 0 ? 1 : 0); }   // b > 0

// Whether pages of a layer of a and of one of b, which begins `by` behind it, meet.
bool rows_meet(const Box& a, const Box& b, Wide by) {
  if (by >= a.row() || -by >= b.row()) return false;
  if (a.n > 1 && b.n > 1 && a.stride != b.stride) return true;   // (not looked into)
  const Wide stride = a.n > 1 ? a.stride : b.stride;
  if (stride == 0) return true;
  // some page j of b and i of a with -b.bytes < by + (j - i) stride < a.bytes
  const Wide lo = floor_div(-by - b.bytes, stride) + 1, hi = -floor_div(by - a.bytes, stride) - 1;
  return std::max<Wide>(lo, 1 - a.n) <= std::min<Wide>(hi, b.n - 1);
}

bool meet(const Box& a, const Box& b) {
  if (a.empty() || b.empty() || a.at >= b.end() || b.at >= a.end()) return false;
  if (a.layers == 1 || b.layers == 1 || a.layer_stride == b.layer_stride) {
    const Wide stride = a.layers > 1 ? a.layer_stride : b.layer_stride;
    for (int64_t d = 1 - a.layers; d < b.layers; ++d)
      if (rows_meet(a, b, b.at - a.at + d * stride)) return true;
    return false;
  }
  if (a.layers * b.layers > 1 << 22) return true;   // (not looked into)
  for (int64_t i = 0; i < a.layers; ++i)
    for (int64_t j = 0; j < b.layers; ++j)
      if (rows_meet(a, b, b.at + j * b.layer_stride - a.at - i * a.layer_stride)) return true;
  return false;
}

// Whether two pages of one pool meet.
bool meets_itself(Box a) {
  if (a.empty()) return false;
  if ((a.n > 1 && a.stride < a.bytes) || (a.layers > 1 && a.layer_stride < a.bytes)) return true;
  if (a.layers == 1 || a.n == 1 || a.layer_stride >= a.row() || a.stride >= a.layer_stride * (a.layers - 1) + a.bytes) return false;
  if (Wide{a.layers} * a.n * a.bytes > a.end() - a.at) return true;
  if (a.n < a.layers) std::swap(a.n, a.layers), std::swap(a.stride, a.layer_stride);
  for (int64_t d = 1; d < a.layers; ++d)
    if (rows_meet(a, a, d * a.layer_stride)) return true;
  return false;
}

// Whether the arrays that a call writes are apart from each other and from what it reads.
int check_apart(const Part* in, int n_in, const Part* out, int n_out, const char* who) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (meet(out[i], in[j])) return operator_fail(KVPRM_EINVAL, "%s: an output overlaps an input", who);
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return operator_fail(KVPRM_EINVAL, "%s: two outputs overlap", who);
  }
  for (int i = 0; i < n_in; ++i)
    if (in[i].bytes > 0 && (!in[i].p || !aligned(in[i].p, 4))) return operator_fail(KVPRM_EINVAL, "%s: an input is NULL or not aligned", who);
  for (int i = 0; i < n_out; ++i)
    if (out[i].bytes > 0 && (!out[i].p || !aligned(out[i].p, 4))) return operator_fail(KVPRM_EINVAL, "%s: an output is NULL or not aligned", who);
  return KVPRM_OK;
}

int check_sizes(int64_t n_pages, int n_pools, int n_seqs, int max_blocks, int n_new, int width, const char* who) {
  if (n_pools < 0 || n_pools > KVPRM_MAX_POOLS) return operator_fail(KVPRM_EINVAL, "%s: %d pools (at most %d)", who, n_pools, KVPRM_MAX_POOLS);
  if (n_pages < 0 || n_pages > (int64_t{1} << 30))
    return operator_fail(KVPRM_EINVAL, "%s: n_pages %lld", who, static_cast<long long>(n_pages));
  if (n_seqs < 0 || max_blocks < 0 || n_new < 0 || width < 0)
    return operator_fail(KVPRM_EINVAL, "%s: n_seqs %d, max_blocks %d, n_new %d, width %d", who, n_seqs, max_blocks, n_new, width);
  if (n_seqs > KVPRM_MAX_SEQS || n_new > KVPRM_MAX_SEQS || max_blocks > kMost || width > kMost)
    return operator_fail(KVPRM_EINVAL, "%s: more than %d sequences, or block tables of more than %d pages", who, KVPRM_MAX_SEQS, kMost);
  if (static_cast<int64_t>(n_new) * width > 0x3FFFFFFF)   // pages that may be wanted: 30 bits, and one for the copy
    return operator_fail(KVPRM_EINVAL, "%s: %d block tables of %d pages", who, n_new, width);
  return KVPRM_OK;
}

int check_pools(const kvprm_pool* pools, int n, int64_t n_pages, CopyLaunch<KVPRM_MAX_POOLS>* c, const char* who) {
  if (n > 0 && !pools) return operator_fail(KVPRM_EINVAL, "%s: no pools", who);
  int64_t pieces = 0;
  c->n_pools = n;
  for (int k = 0; k < n; ++k) {
    const kvprm_pool& p = pools[k];
    if (p.layers < 0 || p.page_bytes < 0 || p.page_bytes > 0x7FFFFFFF || p.page_bytes % 16 || p.layer_stride % 16 || p.page_stride % 16)
      return operator_fail(KVPRM_EINVAL, "%s: pool %d has %d layers of pages of %lld bytes, %lld and %lld apart (multiples of 16)", who, k,
                           p.layers, static_cast<long long>(p.page_bytes), static_cast<long long>(p.layer_stride), static_cast<long long>(p.page_stride));
    if (n_pages > 0 && p.layers > 0 && p.page_bytes > 0 && (!p.base || !aligned(p.base, 16)))
      return operator_fail(KVPRM_EINVAL, "%s: pool %d is NULL or not 16-byte aligned", who, k);
    c->pool[k] = p;
    c->first[k] = static_cast<int32_t>(pieces);
    pieces += static_cast<int64_t>((p.page_bytes + kPiece - 1) / kPiece) * p.layers;
    if (pieces > 0x7FFFFFFF) return operator_fail(KVPRM_EINVAL, "%s: pages of all layers are too large", who);
  }
  c->first[n] = static_cast<int32_t>(pieces);
  return KVPRM_OK;
}

// Whether the pages that a call copies are apart from each other, from its arrays and from its workspace, and that from the arrays.
int check_pages_apart(const kvprm_pool* pools, int n, int64_t n_pages, const Part* in, int n_in, const Part* out, int n_out, const Part& workspace,
                      const char* who) {
  struct Place {
    Box box;
    int k;   // pool, or -1
  };
  Place places[KVPRM_MAX_POOLS + 16];
  int count = 0;
  for (int k = 0; k < n; ++k) {
    const Box box(pools[k], n_pages);
    if (meets_itself(box)) return operator_fail(KVPRM_EINVAL, "%s: pages of pool %d overlap", who, k);
    if (!box.empty()) places[count++] = {box, k};
  }
  auto add = [&](const Part& p) {
    if (p.bytes > 0) places[count++] = {Box(p), -1};
  };
  for (int i = 0; i < n_in; ++i) {
    if (meet(workspace, in[i])) return operator_fail(KVPRM_EINVAL, "%s: the workspace overlaps an input", who);
    add(in[i]);
  }
  for (int i = 0; i < n_out; ++i) {
    if (meet(workspace, out[i])) return operator_fail(KVPRM_EINVAL, "%s: the workspace overlaps an output", who);
    add(out[i]);
  }
  add(workspace);
  std::sort(places, places + count, [](const Place& a, const Place& b) { return a.box.at < b.box.at; });
  for (int i = 0; i < count; ++i)
    for (int j = i + 1; j < count && places[j].box.at < places[i].box.end(); ++j) {
      const Place &a = places[i], &b = places[j];
      if ((a.k < 0 && b.k < 0) || !meet(a.box, b.box)) continue;
      if (a.k < 0 || b.k < 0) return operator_fail(KVPRM_EINVAL, "%s: pool %d overlaps another argument", who, std::max(a.k, b.k));
      return operator_fail(KVPRM_EINVAL, "%s: pools %d and %d overlap", who, std::min(a.k, b.k), std::max(a.k, b.k));
    }
  return KVPRM_OK;
}

// `most`: pages that may be copied; `entries`: of the tables.  One launch where both are few: a launch among others takes 8 us of a
// stream's time, so a step of 16 sequences 9 instead of 16, while the cluster copies 4 MB in 8.
template <typename T>
cudaError_t launch(const CopyLaunch<KVPRM_MAX_POOLS>& c, const T& t, int64_t most, int64_t entries, cudaStream_t stream) {
  const int64_t pieces = c.first[c.n_pools] * most, work = std::max(pieces, (entries + 127) / 128);   // of warps
  CopyLaunch<kFewPools> few;
  few.n_pools = std::min(c.n_pools, kFewPools);
  for (int k = 0; k < few.n_pools; ++k) few.pool[k] = c.pool[k];
  for (int k = 0; k <= few.n_pools; ++k) few.first[k] = c.first[k];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCluster);   // (the kernel's own cluster size)
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  if (c.n_pools <= kFewPools && work <= kSmall) return cudaLaunchKernelEx(&cfg, small_kernel<T>, few, t);
  cudaError_t e = cudaLaunchKernelEx(&cfg, plan_kernel<T>, t);
  int dev = 0, sms = 0;
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess || work == 0) return e;   // (no tables, no copies)
  cfg.gridDim = dim3(static_cast<unsigned>(std::min<int64_t>((work + kCopyThreads / 32 - 1) / (kCopyThreads / 32), int64_t{sms} * kCopyCtas)));
  cfg.blockDim = dim3(kCopyThreads);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return c.n_pools <= kFewPools ? cudaLaunchKernelEx(&cfg, copy_kernel<kFewPools, T>, few, t)
                                : cudaLaunchKernelEx(&cfg, copy_kernel<KVPRM_MAX_POOLS, T>, c, t);
}

int64_t fork_bytes(const kvprm_fork& f) {
  return 256 + 2 * round_up(4 * f.n_pages) + round_up(16 * int64_t{f.n_new}) + round_up(8 * int64_t{f.n_new});
}
int64_t compact_bytes(const kvprm_compact& f) { return 4 * round_up(4 * f.n_pages) + 256; }

int check_fork(const kvprm_fork* f, const char* who) {
  if (!f) return operator_fail(KVPRM_EINVAL, "%s: no arguments", who);
  return check_sizes(f->n_pages, f->n_pools, f->n_seqs, f->max_blocks, f->n_new, f->width, who);
}
int check_compact(const kvprm_compact* f, const char* who) {
  if (!f) return operator_fail(KVPRM_EINVAL, "%s: no arguments", who);
  return check_sizes(f->n_pages, f->n_pools, f->n_seqs, f->max_blocks, 0, 0, who);
}
int check_workspace(const void* workspace, int64_t bytes, int64_t need, const char* who) {
  if (!workspace || !aligned(workspace, 256)) return operator_fail(KVPRM_EINVAL, "%s: workspace is NULL or not 256-byte aligned", who);
  if (bytes < need)
    return operator_fail(KVPRM_ECAPACITY, "%s: a workspace of %lld bytes, %lld needed", who, static_cast<long long>(bytes), static_cast<long long>(need));
  return KVPRM_OK;
}

struct Scratch {
  uint8_t* p;
  template <typename T>
  T* take(int64_t n) {
    T* const r = reinterpret_cast<T*>(p);
    p += round_up(n * static_cast<int64_t>(sizeof(T)));
    return r;
  }
};

}  // namespace

}  // namespace kvprm

using namespace kvprm;

extern "C" {

int kvprm_fork_workspace(const kvprm_pool*, const kvprm_fork* f, int64_t* bytes) {
  const char* who = "kvprm_fork_workspace";
  if (!bytes) return operator_fail(KVPRM_EINVAL, "%s: bytes is NULL", who);
  if (const int rc = check_fork(f, who)) return rc;
  *bytes = fork_bytes(*f);
  return KVPRM_OK;
}

int kvprm_cache_fork(const kvprm_pool* pools, const kvprm_fork* f, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* who = "kvprm_cache_fork";
  if (const int rc = check_fork(f, who)) return rc;
  CopyLaunch<KVPRM_MAX_POOLS> c;
  if (const int rc = check_pools(pools, f->n_pools, f->n_pages, &c, who)) return rc;
  const int64_t table = 4 * int64_t{f->n_seqs} * f->max_blocks;
  const Part in[] = {{f->refs, 4 * f->n_pages}, {f->block_table, table}, {f->lens, 4 * int64_t{f->n_seqs}},
                     {f->parents, 4 * int64_t{f->n_new}}, {f->room, f->room ? 4 * int64_t{f->n_new} : 0}};
  const Part out[] = {{f->refs_out, 4 * f->n_pages}, {f->table_out, 4 * int64_t{f->n_new} * f->width},
                      {f->lens_out, 4 * int64_t{f->n_new}}, {f->counts, 8}};
  if (const int rc = check_apart(in, 5, out, 4, who)) return rc;
  if (const int rc = check_workspace(workspace, workspace_bytes, fork_bytes(*f), who)) return rc;
  if (const int rc = check_pages_apart(pools, f->n_pools, f->n_pages, in, 5, out, 4, {workspace, fork_bytes(*f)}, who)) return rc;
  ForkLaunch a;
  a.f = *f;
  Scratch w{static_cast<uint8_t*>(workspace)};
  a.count = w.take<int32_t>(2);
  a.first = w.take<int32_t>(f->n_pages);
  a.free_pages = w.take<int32_t>(f->n_pages);
  a.rows = w.take<int4>(f->n_new);
  a.pairs = w.take<int2>(f->n_new);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = launch(c, a, f->n_new, int64_t{f->n_new} * f->width, st);
  return e == cudaSuccess ? KVPRM_OK : operator_fail(KVPRM_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

int kvprm_compact_workspace(const kvprm_pool*, const kvprm_compact* f, int64_t* bytes) {
  const char* who = "kvprm_compact_workspace";
  if (!bytes) return operator_fail(KVPRM_EINVAL, "%s: bytes is NULL", who);
  if (const int rc = check_compact(f, who)) return rc;
  *bytes = compact_bytes(*f);
  return KVPRM_OK;
}

int kvprm_cache_compact(const kvprm_pool* pools, const kvprm_compact* f, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* who = "kvprm_cache_compact";
  if (const int rc = check_compact(f, who)) return rc;
  CopyLaunch<KVPRM_MAX_POOLS> c;
  if (const int rc = check_pools(pools, f->n_pools, f->n_pages, &c, who)) return rc;
  const int64_t table = 4 * int64_t{f->n_seqs} * f->max_blocks;
  const Part in[] = {{f->refs, 4 * f->n_pages}, {f->block_table, table}, {f->lens, 4 * int64_t{f->n_seqs}}};
  const Part out[] = {{f->refs_out, 4 * f->n_pages}, {f->table_out, table}, {f->moved, 4 * f->n_pages}, {f->counts, 8}};
  if (const int rc = check_apart(in, 3, out, 4, who)) return rc;
  if (const int rc = check_workspace(workspace, workspace_bytes, compact_bytes(*f), who)) return rc;
  if (const int rc = check_pages_apart(pools, f->n_pools, f->n_pages, in, 3, out, 4, {workspace, compact_bytes(*f)}, who)) return rc;
  CompactLaunch a;
  a.f = *f;
  Scratch w{static_cast<uint8_t*>(workspace)};
  a.count = w.take<int32_t>(1);
  a.low = w.take<int32_t>(f->n_pages);
  a.high = w.take<int32_t>(f->n_pages);
  a.pairs = w.take<int2>(f->n_pages);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = launch(c, a, f->n_pages / 2, int64_t{f->n_seqs} * f->max_blocks, st);
  return e == cudaSuccess ? KVPRM_OK : operator_fail(KVPRM_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

}  // extern "C"
