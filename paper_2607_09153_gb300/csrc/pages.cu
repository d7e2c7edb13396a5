// The pages' bookkeeping between two steps of a search: kvprm_cache_fork (sequences dropped, doubled and given room) and
// kvprm_cache_compact (pages in use moved to the pool's beginning).
//
// Either is two launches.  The first works out tables, references and who is copied where: one cluster of CTAs, whose
// barrier separates the steps, because each step needs what all threads found in the one before and the whole is a few
// thousand to a few hundred thousand numbers.  The second copies pages, warp by warp in pieces of 4 KB, over all layers of
// all pools; it is launched beside the first one's end and learns there how many there are.  Nothing is decided by who
// comes first: counts are sums, of several that want a page the lowest sequence has it, free pages go by their numbers.
#include <cuda_runtime.h>

#include <algorithm>

#include "ptx.cuh"
#include "rope.h"

namespace kvprm {

namespace {

constexpr int kThreads = 1024, kCluster = 8;
constexpr int kCopyCtas = 8;       // of an SM
constexpr int kMost = 1 << 24;     // sequences, and pages of a block table
constexpr int kPage = 16, kNobody = 0x7FFFFFFF;
constexpr int kCopyThreads = 256, kCopyUnroll = 8, kPiece = 32 * 16 * kCopyUnroll;   // of a warp: 4 KB

// ---------------------------------------------------------------- copying
struct CopyLaunch {
  kvprm_pool pool[KVPRM_MAX_POOLS];
  int32_t first[KVPRM_MAX_POOLS + 1];   // pieces of a page of the pools before
  int32_t n_pools;
  const int32_t* count;                 // of pages to copy
  const int2* pairs;                    // from, to
};

__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyLaunch a) {
  grid_dep_wait();
  const int lane = threadIdx.x & 31;
  const int per_copy = a.first[a.n_pools];
  const int64_t items = static_cast<int64_t>(__ldcg(a.count)) * per_copy;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kCopyThreads / 32);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kCopyThreads / 32) + (threadIdx.x >> 5); i < items; i += step) {
    const int64_t j = i / per_copy;
    int r = static_cast<int>(i - j * per_copy), k = 0;
    while (r >= a.first[k + 1]) ++k;
    r -= a.first[k];
    const kvprm_pool& p = a.pool[k];
    const int pieces = static_cast<int>((p.page_bytes + kPiece - 1) / kPiece), layer = r / pieces, piece = r - layer * pieces;
    const int2 pair = __ldcg(a.pairs + j);
    uint8_t* base = static_cast<uint8_t*>(p.base) + layer * p.layer_stride + static_cast<int64_t>(piece) * kPiece + lane * 16;
    if (pair.y < 0) continue;   // no page was free
    const uint8_t* src = base + pair.x * p.page_stride;
    uint8_t* dst = base + pair.y * p.page_stride;
    const int64_t left = p.page_bytes - static_cast<int64_t>(piece) * kPiece - lane * 16;   // bytes from this lane's first on
    uint4 v[kCopyUnroll];
#pragma unroll
    for (int x = 0; x < kCopyUnroll; ++x)
      if (x * 512 < left) v[x] = __ldcs(reinterpret_cast<const uint4*>(src + x * 512));
#pragma unroll
    for (int x = 0; x < kCopyUnroll; ++x)
      if (x * 512 < left) *reinterpret_cast<uint4*>(dst + x * 512) = v[x];
  }
}

// ---------------------------------------------------------------- a cluster's steps
__device__ __forceinline__ int cluster_thread() { return static_cast<int>(cluster_rank()) * kThreads + threadIdx.x; }
constexpr int kAll = kCluster * kThreads;

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

// The sum of a value over the CTA's threads; in all of them.
__device__ __forceinline__ uint64_t cta_sum(uint64_t v, uint64_t* s_warp) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  __syncthreads();   // (the last use's sums have been read)
  if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
  __syncthreads();
  uint64_t sum = s_warp[threadIdx.x & 31];
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  return sum;
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
  __syncthreads();
  if (lane == 31) s_warp[threadIdx.x >> 5] = scan;
  __syncthreads();
  uint64_t sum = s_warp[lane], before = lane < static_cast<int>(threadIdx.x >> 5) ? sum : 0;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, d);
    before += __shfl_xor_sync(0xffffffffu, before, d);
  }
  *total = sum;
  return before + scan - v;
}

// Indices 0 .. n - 1 are shared out as one range a CTA.  sum_of tells the cluster what a CTA's range comes to; after its
// barrier, each_before calls f(index, value, sum of all values before it), and returns the sum of all.
struct Range {
  int lo, hi;
  __device__ __forceinline__ explicit Range(int n) {
    const int per = (n + kCluster - 1) / kCluster;
    lo = min(n, per * static_cast<int>(cluster_rank()));
    hi = min(n, lo + per);
  }
};
template <typename V>
__device__ __forceinline__ void sum_of(int n, V value, uint64_t* told, uint64_t* s_warp) {
  const Range r(n);
  uint64_t sum = 0;
  for (int i = r.lo + threadIdx.x; i < r.hi; i += kThreads) sum += value(i);
  sum = cta_sum(sum, s_warp);
  if (threadIdx.x == 0) tell(told, sum);
}
template <typename V, typename F>
__device__ __forceinline__ void each_before(int n, V value, F f, const uint64_t* told, uint64_t* s_warp) {
  const Range r(n);
  uint64_t carry = 0, total;
  for (uint32_t i = 0; i < cluster_rank(); ++i) carry += told[i];
  for (int i0 = r.lo; i0 < r.hi; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const uint64_t v = i < r.hi ? value(i) : 0;
    const uint64_t before = cta_before(v, s_warp, &total);
    if (i < r.hi) f(i, v, carry + before);
    carry += total;
  }
}
__device__ __forceinline__ uint64_t sum_told(const uint64_t* told) {
  uint64_t sum = 0;
  for (int i = 0; i < kCluster; ++i) sum += told[i];
  return sum;
}

// Calls f(row, begin, end, lane) for each row of a table in segments of 512 entries, a warp each.
template <typename F>
__device__ __forceinline__ void each_segment(int rows, int width, F f) {
  constexpr int kSegment = 512;
  const int per_row = (width + kSegment - 1) / kSegment, lane = threadIdx.x & 31;
  for (int64_t i = cluster_thread() >> 5; i < static_cast<int64_t>(rows) * per_row; i += kAll / 32) {
    const int row = static_cast<int>(i / per_row), begin = static_cast<int>(i - static_cast<int64_t>(row) * per_row) * kSegment;
    f(row, begin, min(width, begin + kSegment), lane);
  }
}

// ---------------------------------------------------------------- fork
constexpr int32_t kCopied = 1 << 30;   // beside a sequence's place among the free pages: the first is its copy's
struct ForkLaunch {
  kvprm_fork f;
  int32_t *children, *first, *free_pages, *at, *count;   // scratch
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
  int32_t parent, len, pages, full, last, end;   // last: the page that it ends inside, -1: none; end: pages that it is to have
  int64_t lacking;                               // pages beyond its table's width
  __device__ __forceinline__ Heir(const kvprm_fork& f, int i) {
    parent = __ldg(f.parents + i);
    if (parent < 0 || parent >= f.n_seqs) parent = -1;
    len = pages = full = 0;
    last = -1;
    bool bad = false;
    if (parent >= 0) {
      const Held h(f, parent);
      len = h.len;
      bad = h.pages == 0 && h.len != 0;
      pages = min(h.pages, f.width);
      full = h.full;
      if (full < pages) {
        last = __ldg(f.block_table + static_cast<int64_t>(parent) * f.max_blocks + full);
        if (last < 0 || last >= f.n_pages) last = -1;
      }
    }
    const int64_t room = f.room ? max(0, __ldg(f.room + i)) : 0;
    const int64_t want = bad ? 0 : (len + room + kPage - 1) / kPage;
    end = static_cast<int32_t>(min(want, static_cast<int64_t>(f.width)));
    end = max(end, pages);
    lacking = max(int64_t{0}, want - max(end, 0));
  }
};

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 1) fork_kernel(const __grid_constant__ ForkLaunch a) {
  __shared__ uint64_t s_warp[32], s_need[kCluster], s_free[kCluster], s_lacking[kCluster];
  const kvprm_fork& f = a.f;
  const int me = cluster_thread();
  const int n_pages = static_cast<int>(f.n_pages);
  grid_dep_launch();
  for (int p = me; p < n_pages; p += kAll) {
    f.refs_out[p] = __ldg(f.refs + p);
    a.first[p] = kNobody;
  }
  for (int s = me; s < f.n_seqs; s += kAll) a.children[s] = 0;
  step();

  // how many continue a sequence, and of those that end inside a page the first
  for (int i = me; i < f.n_new; i += kAll) {
    const Heir h(f, i);
    if (h.parent >= 0) atomicAdd(a.children + h.parent, 1);
    if (h.last >= 0) atomicMin(a.first + h.last, i);
  }
  step();

  // full pages: one reference less, and one more for each that continues the sequence
  each_segment(f.n_seqs, f.max_blocks, [&](int s, int begin, int end, int lane) {
    const Held h(f, s);
    const int heirs = __ldcg(a.children + s);
    const int32_t* row = f.block_table + static_cast<int64_t>(s) * f.max_blocks;
    for (int b = begin + lane; b < min(end, h.pages); b += 32) {
      const int32_t page = __ldg(row + b);
      const int change = (b < h.full && b < f.width ? heirs : 0) - 1;
      if (page >= 0 && page < n_pages && change != 0) atomicAdd(f.refs_out + page, change);
    }
  });
  step();

  // A page that ends inside is kept by the first who ends in it if nobody else holds it, and copied for the others; what
  // nobody holds or ends in is free.
  auto copies = [&](int i, const Heir& h) { return h.last >= 0 && !(__ldcg(f.refs_out + h.last) <= 0 && __ldcg(a.first + h.last) == i); };
  auto need = [&](int i) {   // pages; in the upper half, copies
    const Heir h(f, i);
    const bool copy = copies(i, h);
    return static_cast<uint64_t>(h.end - h.pages + (copy ? 1 : 0)) | static_cast<uint64_t>(copy ? 1 : 0) << 32;
  };
  auto is_free = [&](int p) { return static_cast<uint64_t>(__ldcg(f.refs_out + p) <= 0 && __ldcg(a.first + p) == kNobody ? 1 : 0); };
  sum_of(f.n_new, need, s_need, s_warp);
  sum_of(n_pages, is_free, s_free, s_warp);
  sum_of(f.n_new, [&](int i) { return static_cast<uint64_t>(Heir(f, i).lacking); }, s_lacking, s_warp);
  step();

  const uint64_t needed = sum_told(s_need);
  const int64_t wanted = static_cast<int64_t>(needed & 0xFFFFFFFFu), have = static_cast<int64_t>(sum_told(s_free));
  each_before(f.n_new, need, [&](int i, uint64_t v, uint64_t before) {
    const Heir h(f, i);
    a.at[i] = static_cast<int32_t>(before & 0xFFFFFFFFu) | (v >> 32 ? kCopied : 0);
    if (v >> 32) a.pairs[before >> 32] = make_int2(h.last, static_cast<int32_t>(before & 0xFFFFFFFFu));
    if (h.last >= 0 && (v >> 32) == 0) f.refs_out[h.last] = 1;   // kept
    f.lens_out[i] = h.len;
  }, s_need, s_warp);
  each_before(n_pages, is_free, [&](int p, uint64_t v, uint64_t before) {
    if (!v || static_cast<int64_t>(before) >= wanted) return;
    a.free_pages[before] = p;
    f.refs_out[p] = 1;
  }, s_free, s_warp);
  if (me == 0) {
    f.counts[0] = static_cast<int32_t>(max(int64_t{0}, have - wanted));
    f.counts[1] = static_cast<int32_t>(min(int64_t{kNobody}, max(int64_t{0}, wanted - have) + static_cast<int64_t>(sum_told(s_lacking))));
  }
  if (me == 0) *a.count = static_cast<int32_t>(needed >> 32);
  step();

  auto given = [&](int64_t k) { return k < have ? __ldcg(a.free_pages + k) : -1; };
  for (int j = me; j < static_cast<int>(needed >> 32); j += kAll) a.pairs[j].y = given(__ldcg(&a.pairs[j].y));
  each_segment(f.n_new, f.width, [&](int i, int begin, int end, int lane) {
    const Heir h(f, i);
    const int32_t at = __ldcg(a.at + i), first = at & (kCopied - 1), more = first + (at & kCopied ? 1 : 0);
    const int32_t* row = f.block_table + static_cast<int64_t>(h.parent < 0 ? 0 : h.parent) * f.max_blocks;
    int32_t* out = f.table_out + static_cast<int64_t>(i) * f.width;
    for (int b = begin + lane; b < end; b += 32) {
      int32_t page = -1;
      if (b < h.pages)
        page = b == h.full && (at & kCopied) ? given(first) : __ldg(row + b);
      else if (b < h.end)
        page = given(more + b - h.pages);
      out[b] = page;
    }
  });
}

// ---------------------------------------------------------------- compact
struct CompactLaunch {
  kvprm_compact f;
  int32_t *low, *high, *count;   // scratch: free pages before the first `live`, pages in use behind them
  int2* pairs;
};

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 1) compact_kernel(const __grid_constant__ CompactLaunch a) {
  __shared__ uint64_t s_warp[32], s_live[kCluster], s_below[kCluster];
  const kvprm_compact& f = a.f;
  const int me = cluster_thread(), n_pages = static_cast<int>(f.n_pages);
  grid_dep_launch();
  auto in_use = [&](int p) { return static_cast<uint64_t>(__ldg(f.refs + p) > 0 ? 1 : 0); };
  sum_of(n_pages, in_use, s_live, s_warp);
  step();
  const int live = static_cast<int>(sum_told(s_live));
  // of the first `live` pages, those in use: what is free among them are as many as are in use behind
  sum_of(live, in_use, s_below, s_warp);
  step();
  const int below = static_cast<int>(sum_told(s_below)), moves = live - below;
  each_before(n_pages, in_use, [&](int p, uint64_t used, uint64_t before) {
    const int rank = static_cast<int>(before);   // pages in use before this one
    if (p < live && !used) a.low[p - rank] = p;
    if (p >= live && used) a.high[rank - below] = p;
    if (p < live && used) f.refs_out[p] = __ldg(f.refs + p);
    if (p >= live) f.refs_out[p] = 0;
    f.moved[p] = p < live && used ? p : -1;
  }, s_live, s_warp);
  step();
  for (int j = me; j < moves; j += kAll) {
    const int from = __ldcg(a.high + j), to = __ldcg(a.low + j);
    a.pairs[j] = make_int2(from, to);
    f.moved[from] = to;
    f.refs_out[to] = __ldg(f.refs + from);
  }
  if (me == 0) {
    *a.count = moves;
    f.counts[0] = live;
    f.counts[1] = moves;
  }
  step();
  each_segment(f.n_seqs, f.max_blocks, [&](int s, int begin, int end, int lane) {
    const int32_t len = __ldg(f.lens + s);
    const int64_t pages = len < 0 || static_cast<int64_t>(len) > static_cast<int64_t>(kPage) * f.max_blocks ? 0 : (len + kPage - 1) / kPage;
    for (int b = begin + lane; b < end; b += 32) {
      const int64_t at = static_cast<int64_t>(s) * f.max_blocks + b;
      int32_t page = -1;
      if (b < pages) {
        page = __ldg(f.block_table + at);
        if (page >= 0 && page < n_pages) page = __ldcg(f.moved + page);
      }
      f.table_out[at] = page;
    }
  });
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
  if (n_seqs > kMost || n_new > kMost || max_blocks > kMost || width > kMost)
    return operator_fail(KVPRM_EINVAL, "%s: more than %d sequences, or block tables of more pages", who, kMost);
  if (static_cast<int64_t>(n_new) * width > 0x3FFFFFFF)   // pages that may be wanted: 30 bits, and one for the copy
    return operator_fail(KVPRM_EINVAL, "%s: %d block tables of %d pages", who, n_new, width);
  return KVPRM_OK;
}

int check_pools(const kvprm_pool* pools, int n, int64_t n_pages, CopyLaunch* c, const char* who) {
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

// `most`: pages that may be copied.
cudaError_t launch_copy(const CopyLaunch& c, int64_t most, cudaStream_t stream) {
  const int64_t pieces = c.first[c.n_pools] * most;
  if (pieces == 0) return cudaSuccess;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(std::min<int64_t>((pieces + kCopyThreads / 32 - 1) / (kCopyThreads / 32), int64_t{sms} * kCopyCtas)));
  cfg.blockDim = dim3(kCopyThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, copy_kernel, c);
}

template <typename K, typename A>
cudaError_t launch_cluster(K kernel, const A& a, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCluster);   // (the kernel's own cluster size)
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

int64_t fork_bytes(const kvprm_fork& f) {
  return round_up(4 * int64_t{f.n_seqs}) + 2 * round_up(4 * f.n_pages) + 3 * round_up(4 * int64_t{f.n_new}) + 256;
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
  CopyLaunch c;
  if (const int rc = check_pools(pools, f->n_pools, f->n_pages, &c, who)) return rc;
  const int64_t table = 4 * int64_t{f->n_seqs} * f->max_blocks;
  const Part in[] = {{f->refs, 4 * f->n_pages}, {f->block_table, table}, {f->lens, 4 * int64_t{f->n_seqs}},
                     {f->parents, 4 * int64_t{f->n_new}}, {f->room, f->room ? 4 * int64_t{f->n_new} : 0}};
  const Part out[] = {{f->refs_out, 4 * f->n_pages}, {f->table_out, 4 * int64_t{f->n_new} * f->width},
                      {f->lens_out, 4 * int64_t{f->n_new}}, {f->counts, 8}};
  if (const int rc = check_apart(in, 5, out, 4, who)) return rc;
  if (const int rc = check_workspace(workspace, workspace_bytes, fork_bytes(*f), who)) return rc;
  ForkLaunch a;
  a.f = *f;
  Scratch w{static_cast<uint8_t*>(workspace)};
  a.count = w.take<int32_t>(1);
  a.children = w.take<int32_t>(f->n_seqs);
  a.first = w.take<int32_t>(f->n_pages);
  a.free_pages = w.take<int32_t>(f->n_pages);
  a.at = w.take<int32_t>(f->n_new);
  a.pairs = w.take<int2>(f->n_new);
  c.count = a.count;
  c.pairs = a.pairs;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = launch_cluster(fork_kernel, a, st);
  if (e == cudaSuccess) e = launch_copy(c, f->n_new, st);
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
  CopyLaunch c;
  if (const int rc = check_pools(pools, f->n_pools, f->n_pages, &c, who)) return rc;
  const int64_t table = 4 * int64_t{f->n_seqs} * f->max_blocks;
  const Part in[] = {{f->refs, 4 * f->n_pages}, {f->block_table, table}, {f->lens, 4 * int64_t{f->n_seqs}}};
  const Part out[] = {{f->refs_out, 4 * f->n_pages}, {f->table_out, table}, {f->moved, 4 * f->n_pages}, {f->counts, 8}};
  if (const int rc = check_apart(in, 3, out, 4, who)) return rc;
  if (const int rc = check_workspace(workspace, workspace_bytes, compact_bytes(*f), who)) return rc;
  CompactLaunch a;
  a.f = *f;
  Scratch w{static_cast<uint8_t*>(workspace)};
  a.count = w.take<int32_t>(1);
  a.low = w.take<int32_t>(f->n_pages);
  a.high = w.take<int32_t>(f->n_pages);
  a.pairs = w.take<int2>(f->n_pages);
  c.count = a.count;
  c.pairs = a.pairs;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = launch_cluster(compact_kernel, a, st);
  if (e == cudaSuccess) e = launch_copy(c, f->n_pages / 2, st);
  return e == cudaSuccess ? KVPRM_OK : operator_fail(KVPRM_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

}  // extern "C"
