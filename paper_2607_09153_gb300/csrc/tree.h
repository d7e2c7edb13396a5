// Attention of drafted tokens over the paged cache (internal): what the two kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/kvprm.h"

namespace kvprm {

constexpr int kTreeSeqs = 1024;        // sequences of a launch at most (longer batches take several)
constexpr int kTreePage = 16;

struct TreeLaunch {
  kvprm_tree t;
  const uint8_t* pages;
  const uint8_t* exponents;
  int64_t n_pages;
  int32_t n_kv, group, seq0, n_seqs;   // sequences seq0 .. seq0 + n_seqs - 1
  uint32_t group_m;                    // ceil(2^32 / group), 0 for a group of one (tree_token)
  int32_t whole;                       // 1: no pair is cut; 2: CTA i has pair i (4-bit pages)
  int32_t fill;                        // 1: rows that no sequence writes are written too (tree_fill)
  int32_t weight_full, weight_part;    // places of a block of a pair with all its tiles, or with fewer
  float scale_log2;                    // scores in units of log2
  int32_t* line;                       // [n_seqs + 1], then the CTAs (4-bit pages on registers: the warps) that took part: for the join
  float* part_o;                       // [2 * CTAs][head_dim][rows] (4-bit pages on registers: means, [2 * warps][rows][head_dim])
  float2* part_ml;                     // [2 * CTAs][rows], or [2 * warps][rows]: maxima and sums
};

#ifdef __CUDACC__

// The work of a launch is one line, laid out sequence by sequence, in a sequence (kv head, rows) by (kv head, rows) -- a
// "pair" -- and in a pair block by block (of BLOCK keys), the cached ones first, then those of drafted tokens.  A block takes as
// many places as its time weighs, and a pair begins with the places of LEAD blocks that stand for what it costs to begin
// one.  Each CTA takes an equal share of the line, whatever the lengths are: the blocks whose first place it holds, so at
// most two of its pairs are shared with other CTAs.  Those leave partial results (slot 2 i + 1 of CTA i for a pair
// that begins in its share, 2 i for one that began before), which a second launch joins in order (tree_join.cu).  With
// `whole` set a pair goes to the CTA that holds its first block.  The line's marks come from the device's own lengths (a
// prefix sum over the sequences at the start of each CTA), so that nothing is planned on the host.
struct TreeSeq {
  int32_t len, start, drafts, cached_blocks, blocks, tiles;
  bool bad;        // a length that cannot be: every output NaN
  bool left_out;   // drafts that cannot be
};

template <int ROWS, int BLOCK>
__device__ __forceinline__ TreeSeq tree_seq(const TreeLaunch& a, int s) {
  TreeSeq q;
  q.len = __ldg(a.t.lens + a.seq0 + s);
  q.start = __ldg(a.t.start + a.seq0 + s);
  const int64_t drafts = static_cast<int64_t>(__ldg(a.t.start + a.seq0 + s + 1)) - q.start;
  const bool none = drafts <= 0 || drafts > a.t.max_drafts || q.start < 0 || q.start + drafts > a.t.n_tokens;
  q.drafts = none ? 0 : static_cast<int32_t>(drafts);
  q.left_out = drafts != q.drafts;
  q.bad = q.len < 0 || (static_cast<int64_t>(q.len) + kTreePage - 1) / kTreePage > a.t.max_blocks;
  if (q.bad) q.len = 0;
  q.tiles = (q.drafts * a.group + ROWS - 1) / ROWS;
  q.cached_blocks = (q.len + BLOCK - 1) / BLOCK;
  q.blocks = q.cached_blocks + (q.drafts + BLOCK - 1) / BLOCK;
  return q;
}

// The geometry of a kernel's line: ROWS query rows of a tile, BLOCK keys, pairs of up to TILES tiles, LEAD (above).
template <int ROWS_, int BLOCK_, int TILES_, int LEAD_>
struct TreeGeometry {
  static constexpr int ROWS = ROWS_, BLOCK = BLOCK_, TILES = TILES_, LEAD = LEAD_;
  static constexpr int kSlotRows = ROWS * TILES;   // of a partial result
};

// Places that a block of all of a head's pairs takes.
template <typename G>
__device__ __forceinline__ int32_t tree_width(const TreeLaunch& a, int tiles) {
  return tiles / G::TILES * a.weight_full + (tiles % G::TILES != 0 ? a.weight_part : 0);
}

// Writes the rows of tokens that no sequence has: zeros (they see nothing), or NaN where the sequence is left out.  A warp a
// token, over the launch's CTAs; only where tree_line found that there may be such tokens.
template <int HD>
__device__ __forceinline__ void tree_fill(const TreeLaunch& a) {
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * warps + (threadIdx.x >> 5); t < a.t.n_tokens; t += int64_t{gridDim.x} * warps) {
    bool own = false, lost = false;
    for (int s = lane; s < a.t.n_seqs; s += 32) {
      const int64_t s0 = __ldg(a.t.start + s), s1 = __ldg(a.t.start + s + 1);
      if (t < s0 || t >= s1) continue;
      const bool fine = s1 - s0 <= a.t.max_drafts && s0 >= 0 && s1 <= a.t.n_tokens;
      own = own || fine;
      lost = lost || !fine;
    }
    if (__any_sync(0xffffffffu, own)) continue;
    const uint32_t two = __any_sync(0xffffffffu, lost) ? 0x7FC07FC0u : 0u;
    __nv_bfloat16* row = static_cast<__nv_bfloat16*>(a.t.out) + t * a.t.out_token;
    for (int i = lane; i < a.t.n_q_heads * (HD / 8); i += 32)
      *reinterpret_cast<uint4*>(row + i / (HD / 8) * a.t.out_head + i % (HD / 8) * 8) = make_uint4(two, two, two, two);
  }
}

// off[s] = the first place of sequence s, off[n_seqs] = the line's length (kept below 2^31 by the host).  All threads.
template <typename G, int THREADS, int HD>
__device__ __forceinline__ void tree_line(const TreeLaunch& a, int32_t* off, int32_t* warp_sum) {
  constexpr int kPer = (kTreeSeqs + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.n_seqs + THREADS - 1) / THREADS;   // <= kPer
  int32_t mine[kPer], sum = 0;
  // sequences follow one another from token 0 to the last one, unless one of these says otherwise
  bool gaps = a.n_seqs == 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (k >= per) break;
    const int s = tid * per + k;
    mine[k] = sum;
    if (s < a.n_seqs) {
      const TreeSeq q = tree_seq<G::ROWS, G::BLOCK>(a, s);
      if (q.drafts > 0) sum += (q.blocks + G::LEAD) * tree_width<G>(a, q.tiles) * a.n_kv;
      gaps = gaps || q.left_out || (a.seq0 + s == 0 && q.start != 0) ||
             (a.seq0 + s == a.t.n_seqs - 1 && q.start + q.drafts != a.t.n_tokens);
    }
  }
  int32_t scan = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int32_t up = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += up;
  }
  if (lane == 31) warp_sum[warp] = scan;
  if (__syncthreads_or(gaps && a.fill)) tree_fill<HD>(a);
  int32_t before = scan - sum;
  for (int w = 0; w < warp; ++w) before += warp_sum[w];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (k >= per) break;
    const int s = tid * per + k;
    if (s < a.n_seqs) off[s] = before + mine[k];
    if (s == a.n_seqs - 1) off[a.n_seqs] = before + sum;
  }
  if (a.n_seqs == 0 && tid == 0) off[0] = 0;
  __syncthreads();
}

// The CTAs' shares of the line: the first `more` have least + 1 places, the others `least`.  A share is as long as a block
// (`widest`) at least, so that every CTA between a pair's first and last holds a block of it.
struct TreeShares {
  int32_t ctas, least, more;
  __device__ __forceinline__ TreeShares(int32_t total, int grid, int widest) : ctas(max(1, min(grid, total / widest))) {
    least = total / ctas;
    more = total - least * ctas;
  }
  __device__ __forceinline__ int32_t begin(int cta) const { return least * cta + min(cta, more); }
  __device__ __forceinline__ int owner(int32_t u) const {   // the CTA whose share holds place u
    const int32_t longer = more * (least + 1);
    return u < longer ? u / (least + 1) : more + (u - longer) / least;
  }
};

// A pair, and one CTA's blocks c0 .. c1 - 1 of it.
struct TreePart {
  TreeSeq q;
  int32_t first;      // the place of its first block
  int s, g, tp;       // sequence, kv head, which TILES tiles
  int tiles, weight, c0, c1;
  __device__ __forceinline__ bool whole() const { return c0 == 0 && c1 == q.blocks; }
  __device__ __forceinline__ int32_t place(int block) const { return first + block * weight; }
};

// Walks a CTA's share [u, u_end); s: the sequence to start looking from (tree_find).
template <typename G>
__device__ __forceinline__ bool tree_next(const TreeLaunch& a, const int32_t* off, int32_t& u, int32_t u_end, int& s,
                                          TreePart& p) {
  while (u < u_end) {
    while (u >= off[s + 1]) ++s;
    p.q = tree_seq<G::ROWS, G::BLOCK>(a, s);
    p.s = s;
    const int32_t depth = p.q.blocks + G::LEAD, head = depth * tree_width<G>(a, p.q.tiles), local = u - off[s];
    p.g = local / head;
    p.tp = (local - p.g * head) / (a.weight_full * depth);
    p.tiles = min(G::TILES, p.q.tiles - G::TILES * p.tp);
    p.weight = p.tiles == G::TILES ? a.weight_full : a.weight_part;
    const int32_t pair0 = off[s] + p.g * head + p.tp * a.weight_full * depth;
    p.first = pair0 + G::LEAD * p.weight;
    auto block_at = [&](int32_t place) {   // the first block that begins at a place or after it
      const int32_t d = place - p.first;
      return d <= 0 ? 0 : min(p.q.blocks, (d + p.weight - 1) / p.weight);
    };
    p.c0 = block_at(u);
    p.c1 = block_at(u_end);
    if (a.whole) {
      const bool mine = p.first >= u && p.first < u_end;
      p.c0 = 0;
      p.c1 = mine ? p.q.blocks : 0;
    }
    const int32_t end = pair0 + depth * p.weight;
    u = min(end, u_end);
    if (p.c0 < p.c1) return true;
  }
  return false;
}

// The sequence that holds place u.
__device__ __forceinline__ int tree_find(const int32_t* off, int n, int32_t u) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (off[mid] <= u) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Left for the join by the launch's first CTA.
__device__ __forceinline__ void tree_leave_line(const TreeLaunch& a, const int32_t* off, int ctas) {
  if (blockIdx.x != 0 || a.whole) return;
  for (int i = threadIdx.x; i <= a.n_seqs; i += blockDim.x) a.line[i] = off[i];
  if (threadIdx.x == 0) a.line[a.n_seqs + 1] = ctas;
}

// A row's drafted token: row / group (rows < 2^21, group <= 2^10).
__device__ __forceinline__ int tree_token(const TreeLaunch& a, int row) {
  return a.group_m ? static_cast<int>(__umulhi(static_cast<uint32_t>(row), a.group_m)) : row;
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

// Magnitudes of bf16 numbers as their bits without a sign, which are ordered as the values.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min_s16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.s16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// The larger magnitudes of eight bf16 numbers, as bits, in two halves.
__device__ __forceinline__ uint32_t magnitude2(const uint4& v) {
  return max_u16x2(max_u16x2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), max_u16x2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
}
// The least magnitude of eight that is not zero, plus 0x7FFF, in two halves with a sign: a zero, 0x7FFF, is above all others.
__device__ __forceinline__ uint32_t least2(const uint4& v) {
  auto lifted = [](uint32_t w) { return (w & 0x7FFF7FFFu) + 0x7FFF7FFFu; };
  return min_s16x2(min_s16x2(lifted(v.x), lifted(v.y)), min_s16x2(lifted(v.z), lifted(v.w)));
}
// Whether a row with the largest magnitude `most` and the least one of `least` loses something as fp16 times 2^(142 - e): an element's
// last bit is 2^-7 of its power, and 2^-24 is fp16's.  (One that is not finite has nothing to lose.)
__device__ __forceinline__ bool beyond_f16(uint32_t most, uint32_t least, int e) {
  least ^= 0x80008000u;   // less one
  return most < 0x7F80u && static_cast<int>((min(least & 0xFFFFu, least >> 16) + 1u) >> 7) < e - 32;
}

#endif  // __CUDACC__

// tree.cu: query rows in tiles of 16 (tiles 1) or 32 (tiles 2); CTAs of four warps that run at once on an SM, by the
// registers that a warp's outputs and loads in flight take (four of one tile, with fewer loads in flight, were slower:
// 8 x 32,768 bf16 tokens of 8 kv heads 199 us, three 169).
constexpr int tree_rows_per_sm(int tiles) { return tiles == 2 ? 2 : 3; }
#ifdef __CUDACC__
// A pair's start in blocks (us, one draft over 64 ragged 8-bit sequences: 8 pages 77, 16 75, 32 76; 21 rows of 4 heads over 32
// ragged ones: 8 73, 20 58, 32 58; in chunks, 64 drafts over 16 ragged 8-bit sequences and 21 over 16 bf16 ones: 2 160 and 30,
// 4 162 and 27, 7 167 and 27).
template <int TILES>
using TreeRows = TreeGeometry<16 * TILES, kTreePage, 1, TILES == 1 ? 16 : 20>;
using TreeTc = TreeGeometry<128, 128, 2, 4>;
#endif
cudaError_t launch_tree_rows(const TreeLaunch& a, const kvprm_cache& c, int tiles, int ctas, cudaStream_t stream);
// tree_e2m1.cu: 4-bit pages, tiles of 8, 16 or 32 query rows (tiles of 8: 1, 2 or 4).  Its shares of the line are warps', and it
// joins its partial results itself.
constexpr int kTreeE2m1Warps = 4;   // of a CTA
#ifdef __CUDACC__
template <int NT>
using TreeE2m1 = TreeGeometry<8 * NT, kTreePage, 1, 10>;
#endif
constexpr int tree_e2m1_per_sm(int tiles) { return tiles == 1 ? 3 : 2; }
cudaError_t launch_tree_e2m1(const TreeLaunch& a, const kvprm_cache& c, int tiles, int ctas, cudaStream_t stream);
// tree_tc.cu: in pairs of tiles of 128, on the tensor cores; one CTA on an SM.  The cache has a page at least.
cudaError_t launch_tree_tc(const TreeLaunch& a, const kvprm_cache& c, int ctas, cudaStream_t stream);
// tree_join.cu: joins the partial results that either left; rows: of a partial result (16, 32 or 256).
cudaError_t launch_tree_join(const TreeLaunch& a, const kvprm_cache& c, int rows, cudaStream_t stream);

}  // namespace kvprm
