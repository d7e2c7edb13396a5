// Attention of drafted tokens over the paged cache (internal): what the two kernels share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/kvprm.h"

namespace kvprm {

constexpr int kTreeSeqs = 1024;        // sequences of a launch (longer batches take several)
constexpr int kTreeTickets = 2048;     // the workspace's first words: a counter per CTA, and the last for waits that gave up
constexpr int kTreePage = 16;

struct TreeLaunch {
  kvprm_tree t;
  const uint8_t* pages;
  const uint8_t* exponents;
  int64_t n_pages;
  int32_t n_kv, group, seq0, n_seqs;   // sequences seq0 .. seq0 + n_seqs - 1
  float scale_log2;                    // scores in units of log2
  int32_t* tickets;
  float* part_o;                       // [2 * CTAs][rows][head_dim]
  float2* part_ml;                     // [2 * CTAs][rows]
};

#ifdef __CUDACC__

// The work of a launch is one line of blocks (of kBlock keys), laid end to end: sequence by sequence, in a
// sequence (kv head, tile of ROWS query rows) by (kv head, tile) -- a "pair" -- and in a pair the cached blocks,
// then the blocks of drafted tokens.  CTA i of P takes [W i / P, W (i + 1) / P): equal shares whatever the lengths
// are, with at most two pairs that it shares with other CTAs.  The line's marks come from the device's own lengths
// (a prefix sum over the sequences at the start of each CTA), so that nothing is planned on the host.
struct TreeSeq {
  int32_t len, start, drafts, cached_blocks, blocks, tiles;
  bool bad;   // a length that cannot be: every output NaN
};

template <int ROWS, int BLOCK>
__device__ __forceinline__ TreeSeq tree_seq(const TreeLaunch& a, int s) {
  TreeSeq q;
  q.len = __ldg(a.t.lens + a.seq0 + s);
  q.start = __ldg(a.t.start + a.seq0 + s);
  const int64_t drafts = static_cast<int64_t>(__ldg(a.t.start + a.seq0 + s + 1)) - q.start;
  const bool none = drafts <= 0 || drafts > a.t.max_drafts || q.start < 0 || q.start + drafts > a.t.n_tokens;
  q.drafts = none ? 0 : static_cast<int32_t>(drafts);
  q.bad = q.len < 0 || (static_cast<int64_t>(q.len) + kTreePage - 1) / kTreePage > a.t.max_blocks;
  if (q.bad) q.len = 0;
  q.tiles = (q.drafts * a.group + ROWS - 1) / ROWS;
  q.cached_blocks = (q.len + BLOCK - 1) / BLOCK;
  q.blocks = q.cached_blocks + (q.drafts + BLOCK - 1) / BLOCK;
  return q;
}

// off[s] = the first block of sequence s on the line, off[n_seqs] = W.  All threads of the CTA.
template <int ROWS, int BLOCK, int THREADS>
__device__ __forceinline__ void tree_line(const TreeLaunch& a, int64_t* off, int64_t* warp_sum) {
  constexpr int kPer = (kTreeSeqs + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.n_seqs + THREADS - 1) / THREADS;   // <= kPer
  int64_t mine[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (k >= per) break;
    const int s = tid * per + k;
    mine[k] = sum;
    if (s < a.n_seqs) {
      const TreeSeq q = tree_seq<ROWS, BLOCK>(a, s);
      sum += static_cast<int64_t>(q.blocks) * q.tiles * a.n_kv;
    }
  }
  int64_t scan = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t up = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += up;
  }
  if (lane == 31) warp_sum[warp] = scan;
  __syncthreads();
  int64_t before = scan - sum;
  for (int w = 0; w < warp; ++w) before += warp_sum[w];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (k >= per) break;
    const int s = tid * per + k;
    if (s < a.n_seqs) off[s] = before + mine[k];
    if (s == a.n_seqs - 1) off[a.n_seqs] = before + sum;
  }
  __syncthreads();
}

// The sequence that holds block u of the line.
__device__ __forceinline__ int tree_find(const int64_t* off, int n, int64_t u) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (off[mid] <= u) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// The CTA of P whose share holds block u: the largest i with W i / P <= u.
__device__ __forceinline__ int tree_owner(int64_t u, int64_t total, int p) {
  return static_cast<int>(((u + 1) * p - 1) / total);
}

// Whether row's drafted token `t` of sequence q sees drafted tokens j0 .. j0 + 15 (bits; j0 a multiple of 16).
__device__ __forceinline__ uint32_t tree_sees16(const TreeLaunch& a, const TreeSeq& q, int t, int j0) {
  uint32_t bits;
  if (a.t.mask) {
    bits = (__ldg(a.t.mask + static_cast<int64_t>(q.start + t) * a.t.mask_words + (j0 >> 5)) >> (j0 & 31)) & 0xFFFFu;
  } else {
    const int n = t - j0 + 1;   // a chain: tokens up to t
    bits = n <= 0 ? 0u : n >= 16 ? 0xFFFFu : (1u << n) - 1u;
  }
  const int have = q.drafts - j0;
  return have >= 16 ? bits : bits & ((1u << have) - 1u);
}

#endif  // __CUDACC__

// tree.cu: query rows in tiles of 16; CTAs that run at once on an SM.
constexpr int kTreeRows16PerSm = 3;
cudaError_t launch_tree_rows16(const TreeLaunch& a, const kvprm_cache& c, int ctas, cudaStream_t stream);
// tree_tc.cu: in pairs of tiles of 128, on the tensor cores; one CTA on an SM.  The cache has a page at least.
cudaError_t launch_tree_tc(const TreeLaunch& a, const kvprm_cache& c, int ctas, cudaStream_t stream);

}  // namespace kvprm
