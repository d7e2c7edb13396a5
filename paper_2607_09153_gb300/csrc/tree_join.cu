// Joins the partial results of pairs that several CTAs shared (tree.h): launched beside the attention kernel's end
// (programmatic dependent launch), its CTAs wait for it and then read the partial softmax states of up to 32 rows of a pair,
// lane by row, in the order of the CTAs that left them -- so the result does not depend on who was last.
//
// Why a launch of its own: the CTA that finishes a pair last joined it at first.  A pair of 33 chunks has ten parts of 126
// rows x 128 dims, whose loads then hang on one SM's latency: 40 to 60 us at the end of a call of 16 ragged caches (attend 21
// drafts, 76 us in all).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"
#include "tree.h"

namespace kvprm {

namespace {

constexpr int kThreads = 256;

template <typename G, int HD>
__global__ void __launch_bounds__(kThreads) tree_join_kernel(const __grid_constant__ TreeLaunch a, int groups) {
  constexpr int R = G::kSlotRows;
  constexpr int kLaneRows = R < 32 ? R : 32, kSplit = 32 / kLaneRows;   // lanes over rows, and over dims where rows are few
  constexpr int kDims = HD / 8 / kSplit;                                // of a thread
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // block: (sequence, kv head, group of rows), groups fastest
  const int group = blockIdx.x % groups, head = blockIdx.x / groups, g = head % a.n_kv, s = head / a.n_kv;
  const TreeSeq q = tree_seq<G::ROWS, G::BLOCK>(a, s);
  const int rows = q.drafts * a.group, row0 = group * kLaneRows;
  if (row0 >= rows) {
    if (blockIdx.x == 0) grid_dep_wait();   // no launch of this kernel ends before the attention kernel
    return;
  }
  const int tp = row0 / R;
  grid_dep_wait();
  const int32_t off = __ldcg(a.line + s), total = __ldcg(a.line + a.n_seqs), ctas = __ldcg(a.line + a.n_seqs + 1);
  const TreeShares shares(total, ctas, 1);
  const int weight = q.tiles - G::TILES * tp >= G::TILES ? a.weight_full : a.weight_part, depth = q.blocks + G::LEAD;
  const int32_t first = off + depth * (g * tree_width<G>(a, q.tiles) + tp * a.weight_full) + G::LEAD * weight;
  const int i0 = shares.owner(first), i1 = shares.owner(first + (q.blocks - 1) * weight);
  if (i0 == i1) return;   // whole: written by its CTA
  const int r = row0 - tp * R + lane % kLaneRows, d0 = warp * (HD / 8) + lane / kLaneRows * kDims;
  float best = -INFINITY, sum = 0.f, o[kDims];
#pragma unroll
  for (int k = 0; k < kDims; ++k) o[k] = 0.f;
#pragma unroll 2
  for (int i = i0; i <= i1; ++i) {
    const int64_t slot = i == i0 ? 2 * i + 1 : 2 * i;
    const float2 ml = __ldcg(a.part_ml + slot * R + r);
    float v[kDims];
#pragma unroll
    for (int k = 0; k < kDims; ++k) v[k] = __ldcg(a.part_o + (slot * HD + d0 + k) * R + r);
    const float now = fmaxf(best, ml.x);   // -infinity: nothing seen so far (a sum of zero, or NaN)
    const float f = best == -INFINITY ? 0.f : ex2_ftz(best - now), e = ml.x == -INFINITY ? 0.f : ex2_ftz(ml.x - now);
    best = now;
    sum = sum * f + ml.y * e;
#pragma unroll
    for (int k = 0; k < kDims; ++k) o[k] = o[k] * f + v[k] * e;
  }
  const int row = tp * R + r;
  if (row >= rows) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that saw nothing: zeros
  const int tok = tree_token(a, row);
  __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.t.out) + (q.start + static_cast<int64_t>(tok)) * a.t.out_token +
                       (g * a.group + row - tok * a.group) * a.t.out_head + d0;
  uint32_t w[kDims / 2];
#pragma unroll
  for (int k = 0; k < kDims / 2; ++k) w[k] = pack_bf16(o[2 * k] * inv, o[2 * k + 1] * inv);
#pragma unroll
  for (int k = 0; k < kDims / 2; k += 2) *reinterpret_cast<uint2*>(dst + 2 * k) = make_uint2(w[k], w[k + 1]);
}

template <typename G, int HD>
cudaError_t launch(const TreeLaunch& a, cudaStream_t stream) {
  const int lane_rows = G::kSlotRows < 32 ? G::kSlotRows : 32;
  const int groups = (a.t.max_drafts * a.group + lane_rows - 1) / lane_rows;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(static_cast<int64_t>(a.n_seqs) * a.n_kv * groups));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, tree_join_kernel<G, HD>, a, groups);
}

}  // namespace

cudaError_t launch_tree_join(const TreeLaunch& a, const kvprm_cache& c, int rows, cudaStream_t stream) {
  const bool wide = c.head_dim == 128;
  if (rows == TreeTc::kSlotRows) return wide ? launch<TreeTc, 128>(a, stream) : launch<TreeTc, 64>(a, stream);
  if (rows == 32) return wide ? launch<TreeRows<2>, 128>(a, stream) : launch<TreeRows<2>, 64>(a, stream);
  return wide ? launch<TreeRows<1>, 128>(a, stream) : launch<TreeRows<1>, 64>(a, stream);
}

}  // namespace kvprm
