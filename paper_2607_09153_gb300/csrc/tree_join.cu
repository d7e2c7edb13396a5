// Joins the partial results of pairs that several CTAs shared (tree.h): launched beside the attention kernel's end
// (programmatic dependent launch), its CTAs wait for it and then read the partial softmax states of up to 32 rows of a pair,
// lane by row, in the order of the CTAs that left them -- so the result does not depend on who was last.
//
// Why a launch of its own: the CTA that finishes a pair last joined it at first.  A pair of 33 chunks has ten parts of 126
// rows x 128 dims, whose loads then hang on one SM's latency: 40 to 60 us at the end of a call of 16 ragged caches (attend 21
// drafts, 76 us in all).
//
// What bounds it: latency.  A thread has 8 dims of a row, four parts' loads in flight, and its CTA is small enough to be
// resident beside the attention kernel's: 6 us for that call.  (With 16 dims, two parts and 256 threads, which had to
// wait for the attention kernel's CTAs to leave, 12.)
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"
#include "tree.h"

namespace kvprm {

namespace {

constexpr int kThreads = 128;
constexpr int kQuarters = 4;   // of the head's dimensions
constexpr int kAhead = 4;      // partial results in flight

template <typename G, int HD>
__global__ void __launch_bounds__(kThreads, 7) tree_join_kernel(const __grid_constant__ TreeLaunch a, int groups, int split) {
  constexpr int R = G::kSlotRows;
  constexpr int kLaneRows = R < 32 ? R : 32, kSplit = 32 / kLaneRows;   // lanes over rows, and over dims where rows are few
  constexpr int kWarpDims = HD / kQuarters / (kThreads / 32), kDims = kWarpDims / kSplit;   // kDims: of a thread
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // block: (sequence, kv head, group of rows, one of `split` shares of the dims), shares fastest
  const int block = blockIdx.x / split, share = blockIdx.x - block * split;
  const int group = block % groups, head = block / groups, g = head % a.n_kv, s = head / a.n_kv;
  const TreeSeq q = tree_seq<G::ROWS, G::BLOCK>(a, s);
  const int rows = q.drafts * a.group, row0 = group * kLaneRows;
  if (row0 >= rows) {
    if (blockIdx.x == 0) grid_dep_wait();   // no launch of this kernel ends before the attention kernel
    return;
  }
  const int tp = row0 / R, r = row0 - tp * R + lane % kLaneRows, row = tp * R + r;
  const int weight = q.tiles - G::TILES * tp >= G::TILES ? a.weight_full : a.weight_part, depth = q.blocks + G::LEAD;
  const int tok = tree_token(a, row);
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.t.out) + (q.start + static_cast<int64_t>(tok)) * a.t.out_token +
                       (g * a.group + row - tok * a.group) * a.t.out_head;
  grid_dep_wait();
  const int32_t off = __ldcg(a.line + s), total = __ldcg(a.line + a.n_seqs), ctas = __ldcg(a.line + a.n_seqs + 1);
  const TreeShares shares(total, ctas, 1);
  const int32_t first = off + depth * (g * tree_width<G>(a, q.tiles) + tp * a.weight_full) + G::LEAD * weight;
  const int i0 = shares.owner(first), i1 = shares.owner(first + (q.blocks - 1) * weight);
  if (i0 == i1) return;   // whole: written by its CTA
  for (int quarter = share; quarter < kQuarters; quarter += split) {
    const int d0 = (quarter * (kThreads / 32) + warp) * kWarpDims + lane / kLaneRows * kDims;
    float best = -INFINITY, sum = 0.f, o[kDims];
#pragma unroll
    for (int k = 0; k < kDims; ++k) o[k] = 0.f;
#pragma unroll 1
    for (int i = i0; i <= i1; i += kAhead) {
      float2 ml[kAhead];
      float v[kAhead][kDims];
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        const int64_t slot = i + x == i0 ? 2 * i0 + 1 : 2 * min(i + x, i1);
        ml[x] = __ldcg(a.part_ml + slot * R + r);
#pragma unroll
        for (int k = 0; k < kDims; ++k) v[x][k] = __ldcg(a.part_o + (slot * HD + d0 + k) * R + r);
      }
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        if (i + x > i1) break;
        const float now = fmaxf(best, ml[x].x);   // -infinity: nothing seen so far (a sum of zero, or NaN)
        const float f = best == -INFINITY ? 0.f : ex2_ftz(best - now), e = ml[x].x == -INFINITY ? 0.f : ex2_ftz(ml[x].x - now);
        best = now;
        sum = sum * f + ml[x].y * e;
#pragma unroll
        for (int k = 0; k < kDims; ++k) o[k] = o[k] * f + v[x][k] * e;
      }
    }
    if (row >= rows) continue;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that saw nothing: zeros
    constexpr int kStep = kDims < 4 ? 2 : 4;
#pragma unroll
    for (int k = 0; k < kDims; k += kStep) {
      const uint32_t lo = pack_bf16(o[k] * inv, o[k + 1] * inv);
      if constexpr (kStep == 2)
        *reinterpret_cast<uint32_t*>(out + d0 + k) = lo;
      else
        *reinterpret_cast<uint2*>(out + d0 + k) = make_uint2(lo, pack_bf16(o[k + 2] * inv, o[k + 3] * inv));
    }
  }
}

template <typename G, int HD>
cudaError_t launch(const TreeLaunch& a, cudaStream_t stream) {
  const int lane_rows = G::kSlotRows < 32 ? G::kSlotRows : 32;
  const int groups = (a.t.max_drafts * a.group + lane_rows - 1) / lane_rows;
  cudaLaunchConfig_t cfg = {};
  const int64_t blocks = static_cast<int64_t>(a.n_seqs) * a.n_kv * groups;
  const int split = blocks <= 1024 ? kQuarters : 1;   // few rows: more CTAs, else fewer to start
  cfg.gridDim = dim3(static_cast<unsigned>(blocks * split));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, tree_join_kernel<G, HD>, a, groups, split);
}

}  // namespace

cudaError_t launch_tree_join(const TreeLaunch& a, const kvprm_cache& c, int rows, cudaStream_t stream) {
  const bool wide = c.head_dim == 128;
  if (rows == TreeTc::kSlotRows) return wide ? launch<TreeTc, 128>(a, stream) : launch<TreeTc, 64>(a, stream);
  if (rows == 32) return wide ? launch<TreeRows<2>, 128>(a, stream) : launch<TreeRows<2>, 64>(a, stream);
  return wide ? launch<TreeRows<1>, 128>(a, stream) : launch<TreeRows<1>, 64>(a, stream);
}

}  // namespace kvprm
