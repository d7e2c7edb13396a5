// Attention of drafted tokens over 4-bit pages (e2m1 codes, a power of two for each 32 elements): up to 32 query rows (row =
// drafted token and head of the kv head's group) a tile, by warp-level matrix instructions.
//
// The products are the transposed ones, S^T = K Q^T and O^T = V^T P^T: the cache's rows fill the 16 rows of an instruction
// and the queries its 8 columns, so a plain decoding step (up to 8 query heads on a kv head) takes half the instructions
// that tiles of 16 query rows take.  A lane's 16 bytes of a key row are one block of 32 elements: it converts them (one
// instruction for two codes, to fp16), multiplies them by the block's power of two, and has the operands of eight steps;
// dimensions run in any order as long as Q's follow.  Of the values a lane has the same 16 dimensions of four tokens: the
// nibbles of two tokens are put side by side, so that one conversion gives an operand's pair.  S^T's columns become P^T's
// by one 8 x 8 transposition in registers.
//
// What fp16 lacks in range is kept beside it as powers of two.  A query row is scaled to a largest magnitude of 2^15 to 2^16
// (exact for elements down to 2^-32 of that; rows with smaller ones take their products in bf16, as they are).  A page's key blocks are taken
// relative to a power Ek that its scores are multiplied by in fp32, the values' relative to a power Ev that the outputs are kept
// relative to: blocks from 2^-8 to 2^7 of it are exact.  A page that leaves that window moves Ek or Ev; one whose own
// blocks are further apart takes its products in bf16 instead, whose range is fp32's.  Weights are kept times 2^12, so
// that fp16's steps end at 2^-36 of a full weight's.
//
// Each warp has a share of the work line (tree.h) of its own, copies its pages into a ring in shared memory by itself, two steps
// of two pages ahead, and leaves partial results that a second launch joins: nothing waits at a barrier.  Short pairs stay
// whole instead, a CTA each, whose four warps meet at the end.
//
// What bounds it, measured on a GB300, is instructions: a page of a kv head takes some 295 of a warp (64 conversions, 64
// multiplications by powers, 16 matrix instructions, 16 to put nibbles together, 20 of the softmax, 29 loads and copies), 0.60 of
// the issue slots with the three warps a scheduler that 167 registers leave (ALU pipe 0.47, DRAM 0.53).  One drafted token
// over 8 x 32,768 tokens of 8 heads 63 us (4,530 GB/s), four (16 rows) 83, eight (32 rows) 139; 64 ragged sequences up to 9,001
// of 4 heads 48 us; one sequence of 32,768 of 4 heads 20.  Pages in the general form cost more (the ragged ones / four drafts): a zero
// block in 1,000 56 / 102 us, in 100 72 / 132, blocks 2^26 apart in every page 109 / 252, a query row that fp16 does not hold 103 /
// 237.  Tried: fragments loaded straight into registers, a page ahead (75 us for the first of these: the loads
// share scoreboards) or in single pages (84); four CTAs an SM (81: spills); the next step's scores beside this one's product
// (74); CTAs instead of warps as shares (72; the ragged ones 58, for a part then costs 4 us of barriers); two CTAs of six
// or seven warps (65.6, and 76: spills); a page's scores in two chains of products (the same).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "ptx.cuh"
#include "rope.h"
#include "tree.h"

namespace kvprm {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr float kMargin = 3.f;     // a running maximum may be exceeded by so many powers of two
constexpr float kLift = 12.f;      // weights are times 2^12: 2^(12 + 3) is below 65504
constexpr int kBelow = 8;          // blocks from 2^-8 of E on, to 2^7, are taken in fp16
constexpr int kTop = 239;          // E's field at most: 255, NaN, is never in the window

// 16 bytes into shared memory, in the background.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {   // until all but the last N groups have arrived
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit elements, a row over four lanes, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float power_of(int field) { return __uint_as_float(static_cast<uint32_t>(field) << 23); }
// Whether one of two magnitudes is 2^k or more (field: k + 127; 255: not finite).
__device__ __forceinline__ bool from(uint32_t magnitude, uint32_t field) {
  return max(magnitude & 0xFFFFu, magnitude >> 16) >= field << 7;
}
// Two codes' fp16 times factors, as bf16 (the longer form).
__device__ __forceinline__ uint32_t bf16_times(uint32_t h, float lo, float hi) {
  const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return pack_bf16(v.x * lo, v.y * hi);
}
// The token of a page that row r of S^T, and index r of P V's sums, stand for: a lane's four values' rows are neighbours.
__device__ __forceinline__ int token_of(int r) { return 4 * ((r & 7) >> 1) + (r & 1) + ((r >> 3) << 1); }

// Parts are joined with the weights of their means: a part's sum times 2^(its maximum - top), where top is so far above the
// maximum (by the sum's power, and 2^12 for the number of parts) that all parts' weights together are 1 at most, and the joined sums
// of weights times means finite.  ml: a part's maximum (-infinity: it saw nothing) and sum (0 then; NaN stays NaN).
__device__ __forceinline__ float part_top(const float2& ml) {
  return ml.x + static_cast<float>(static_cast<int>(__float_as_uint(ml.y) >> 23) - 127 + 12);
}
__device__ __forceinline__ float part_weight(const float2& ml, float top) {
  return ml.y * (ml.x == -INFINITY ? 0.f : ex2_ftz(ml.x - top));
}

// A warp's ring of pages: of each a head's keys, values and their exponents.  Rows lie in the order in which the lanes read
// them, so that an access' 128 bytes are in different banks: key row of lane group gid (+ 2 tokens) at 8 n + gid; value row
// 4 c + t at 4 t + c, its 16-byte pieces turned by c >> 1 (the rows are 64 bytes with 128 dims).
template <int HD>
struct Stage {
  static constexpr int kRow = HD / 2, kHead = kTreePage * kRow, kExp = kTreePage * HD / 32;
  static constexpr int kK = 0, kV = kHead, kKe = 2 * kHead, kVe = kKe + kExp, kBytes = kVe + kExp;
};
constexpr int kRing = 4;   // pages of a warp
template <int HD>
constexpr int ring_bytes() { return kWarps * kRing * Stage<HD>::kBytes; }

// NT: tiles of 8 query rows.  WHOLE: no pair is cut.
template <int HD, int NT, bool WHOLE>
__global__ void __launch_bounds__(kThreads, tree_e2m1_per_sm(NT)) tree_e2m1_kernel(const __grid_constant__ TreeLaunch a) {
  using G = TreeE2m1<NT>;
  constexpr int KS = HD / 16;            // 16-dim steps of q . k
  constexpr int MT = HD / 16;            // 16-dim tiles of the output
  constexpr int kW = HD / 32;            // a lane's words of a key row, of eight codes
  constexpr int kVW = HD / 64;           // of each of its four value rows
  constexpr int kRowBytes = HD / 2, kBlocks = HD / 32;
  constexpr int P = 2;                   // pages of a step
  using S = Stage<HD>;
  extern __shared__ __align__(16) uint8_t s_ring[];
  __shared__ int32_t s_off[kTreeSeqs + 1];
  __shared__ int32_t s_sum[kWarps];
  __shared__ uint2 s_q[kWarps][NT][KS][32];   // the scaled queries' fragments, by lane
  __shared__ float2 s_ml[kWarps][8];
  grid_dep_launch();
  tree_line<G, kThreads, HD>(a, s_off, s_sum);
  const int32_t total = s_off[a.n_seqs];
  if (total == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, c = lane & 3;
  // Whole pairs are a CTA's, whose warps take a quarter of the blocks each -- where there is a CTA for each, by its number, for
  // an equal share of the line may hold several short pairs --; else a share is a warp's.
  const TreeShares shares(total, WHOLE ? gridDim.x : gridDim.x * kWarps, a.weight_full);
  const int me = WHOLE ? blockIdx.x : blockIdx.x * kWarps + warp;
  tree_leave_line(a, s_off, shares.ctas);
  const bool direct = WHOLE && a.whole == 2;
  if (!direct && me >= shares.ctas) return;
  constexpr uint32_t head_bytes = kTreePage * kRowBytes, kHeadExp = kTreePage * kBlocks;
  const uint32_t page_bytes = 2 * a.n_kv * head_bytes, page_exp = 2 * a.n_kv * kHeadExp;   // (of 1,024 heads at most)
  // where this lane's pieces of a page go
  uint8_t* const my_ring = s_ring + warp * (kRing * S::kBytes);
  const uint32_t ring = smem_u32(my_ring);
  constexpr int kPer = HD / 32;                       // pieces of a row
  const int row = lane / kPer, piece = lane % kPer;   // (with 128 dims, and 8 rows on)
  const int k_at = S::kK + (8 * ((row & 3) >> 1) + 2 * (row >> 2) + (row & 1)) * kRowBytes + piece * 16;
  const int v_at = S::kV + (4 * (row & 3) + (row >> 2)) * kRowBytes + piece * 16;
  constexpr int k_step = 4 * kRowBytes;
  const int v_step = 2 * kRowBytes + (piece & 2 ? -32 : 32);
  int32_t u = direct ? 0 : shares.begin(me);
  const int32_t u_end = direct ? 1 : shares.begin(me + 1);
  const int head_tiles = (a.t.max_drafts * a.group + G::ROWS - 1) / G::ROWS;   // (direct) CTAs of a kv head
  int s_at = direct ? blockIdx.x / (a.n_kv * head_tiles) : tree_find(s_off, a.n_seqs, u);
  TreePart part;
  auto next_part = [&]() {
    if (!direct) return tree_next<G>(a, s_off, u, u_end, s_at, part);
    if (u++ > 0 || s_at >= a.n_seqs) return false;
    part.q = tree_seq<G::ROWS, G::BLOCK>(a, s_at);
    const int rest = blockIdx.x - s_at * a.n_kv * head_tiles;
    part.g = rest / head_tiles;
    part.tp = rest - part.g * head_tiles;
    part.s = s_at;
    part.first = part.c0 = 0;
    part.tiles = part.weight = 1;
    part.c1 = part.tp < part.q.tiles ? part.q.blocks : 0;
    return part.c1 > 0;
  };
  while (next_part()) {
    const TreeSeq& q = part.q;
    const int g = part.g, row0 = part.tp * G::kSlotRows, rows = q.drafts * a.group;
    const int32_t* table = a.t.block_table + static_cast<int64_t>(a.seq0 + s_at) * a.t.max_blocks;
    const uint8_t* keys = a.pages + g * head_bytes + lane * 16;
    const uint8_t* values = keys + a.n_kv * head_bytes;
    const uint8_t* exps = a.exponents + g * kHeadExp + (lane < static_cast<int>(kHeadExp / 16) ? lane * 16 : a.n_kv * kHeadExp + lane * 16 - kHeadExp);
    // the query rows' elements (HD / 4) c .. of row gid of tile nt
    auto query = [&](int nt) -> const uint4* {
      const int r = row0 + 8 * nt + gid;
      if (r >= rows) return nullptr;
      const int tok = tree_token(a, r);
      return reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.t.q) + (q.start + static_cast<int64_t>(tok)) * a.t.q_token +
                                            (g * a.group + r - tok * a.group) * a.t.q_head + c * (HD / 4));
    };

    // ---- the pages' numbers, a lane each, 32 at a time; 0 for one outside the cache
    const int n_blocks = part.c1 - part.c0;
    const int c0 = WHOLE ? part.c0 + n_blocks * warp / kWarps : part.c0, c1 = WHOLE ? part.c0 + n_blocks * (warp + 1) / kWarps : part.c1;
    const int mine = max(0, min(c1, q.cached_blocks) - c0);
    bool poison = q.bad;        // of all rows of the sequence
    auto ids_of = [&](int k0) {
      const int k = k0 + lane;
      if (k >= mine) return 0;
      const int32_t page = __ldg(table + c0 + k);
      const bool in = page >= 0 && page < a.n_pages;
      poison = poison || !in;
      return in ? page : 0;
    };
    const int pages = a.n_pages > 0 ? mine : 0;   // (an empty pool: every page is outside it)
    int32_t ids = ids_of(0), ids_next = ids_of(32);
    // pages k .. into a step's places of the ring, as far as there are any (a step's are among the same 32)
    auto fetch = [&](int k, uint32_t to) {
#pragma unroll
      for (int y = 0; y < P; ++y) {
        if (k + y >= pages) break;
        const uint32_t page = __shfl_sync(0xffffffffu, ids, (k + y) & 31);
        const uint8_t* from_k = keys + static_cast<uint64_t>(page) * page_bytes;
        const uint8_t* from_v = values + static_cast<uint64_t>(page) * page_bytes;
#pragma unroll
        for (int x = 0; x < S::kHead / 512; ++x) {
          copy16(to + y * S::kBytes + k_at + x * k_step, from_k + x * 512);
          copy16(to + y * S::kBytes + v_at + x * v_step, from_v + x * 512);
        }
        if (lane < 2 * S::kExp / 16) copy16(to + y * S::kBytes + S::kKe + lane * 16, exps + static_cast<uint64_t>(page) * page_exp);
      }
      copies_end();
      if ((k & 31) == 32 - P) {
        ids = ids_next;
        ids_next = ids_of(k + 32 + P);
      }
    };
    struct Loaded {
      uint32_t k[2][kW], v[4][kVW];
      uint32_t ke[2], ve[kBlocks];   // ve: the blocks of four tokens' values
    };
    auto read_keys = [&](int place, Loaded& x) {   // and all exponents
      const uint8_t* at = my_ring + place;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const uint8_t* row = at + S::kK + (8 * n + gid) * kRowBytes + c * (kRowBytes / 4);
        if constexpr (HD == 128) {
          const uint4 r = *reinterpret_cast<const uint4*>(row);
          x.k[n][0] = r.x, x.k[n][1] = r.y, x.k[n][2] = r.z, x.k[n][3] = r.w;
        } else {
          const uint2 r = *reinterpret_cast<const uint2*>(row);
          x.k[n][0] = r.x, x.k[n][1] = r.y;
        }
        x.ke[n] = at[S::kKe + (token_of(gid) + 2 * n) * kBlocks + c * kBlocks / 4];
      }
      const uint8_t* ve = at + S::kVe + 4 * c * kBlocks;
      if constexpr (HD == 128) {
        const uint4 r = *reinterpret_cast<const uint4*>(ve);
        x.ve[0] = r.x, x.ve[1] = r.y, x.ve[2] = r.z, x.ve[3] = r.w;
      } else {
        const uint2 r = *reinterpret_cast<const uint2*>(ve);
        x.ve[0] = r.x, x.ve[1] = r.y;
      }
    };
    auto read_values = [&](int place, Loaded& x) {
      const uint8_t* at = my_ring + place + S::kV;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (HD == 128) {
          const uint2 r = *reinterpret_cast<const uint2*>(at + (4 * t + c) * kRowBytes + ((gid * 8) ^ ((c >> 1) << 5)));
          x.v[t][0] = r.x, x.v[t][1] = r.y;
        } else {
          x.v[t][0] = *reinterpret_cast<const uint32_t*>(at + (4 * t + c) * kRowBytes + gid * 4);
        }
      }
    };
    // the exponents of this lane's block (of its 16 dims) of its four tokens, a byte each
    auto value_bytes = [&](const Loaded& x) {
      if constexpr (HD == 128) {   // word t: token t's four blocks
        const uint32_t sel = (gid >> 1) | (4 + (gid >> 1)) << 4;
        return __byte_perm(__byte_perm(x.ve[0], x.ve[1], sel), __byte_perm(x.ve[2], x.ve[3], sel), 0x5410);
      } else {                     // two tokens' two blocks a word
        return __byte_perm(x.ve[0], x.ve[1], gid & 4 ? 0x7531 : 0x6420);
      }
    };

    // What the part begins with is loaded at once: the pages' numbers, the queries, then the first pages.
    uint4 qv[NT][HD / 32];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint4* src = query(nt);
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) qv[nt][i] = src ? __ldg(src + i) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kRing; k += P) fetch(k, ring + k * S::kBytes);

    // ---- the queries, scaled; a negative scale turns their signs
    float rs[NT][2];   // of rows 2 c and 2 c + 1: the row's power of two times the scores' scale
    bool far = false;  // a row that fp16 does not hold
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      uint32_t most = 0, least = 0x7FFF7FFFu;
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        most = max_u16x2(most, magnitude2(qv[nt][i]));
        least = min_s16x2(least, least2(qv[nt][i]));
      }
      most = max(most & 0xFFFFu, most >> 16);   // (bits without a sign: ordered as the values)
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
      // (2^(142 - e) has to be a normal number; all zero or not finite: any scale does)
      const int e = min(max(static_cast<int>(most >> 7), 15), 254);
      far = far || beyond_f16(most, least, e);
      rs[nt][0] = __shfl_sync(0xffffffffu, power_of(e), 8 * c) * (0x1p-15f * fabsf(a.scale_log2));
      rs[nt][1] = __shfl_sync(0xffffffffu, power_of(e), 8 * c + 4) * (0x1p-15f * fabsf(a.scale_log2));
      const float up = a.scale_log2 < 0.f ? -power_of(269 - e) : power_of(269 - e);
      auto scaled = [&](uint32_t w) { return pack_f16(lo_bf16(w) * up, hi_bf16(w) * up); };
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {   // (read by this lane alone)
        s_q[warp][nt][2 * i][lane] = make_uint2(scaled(qv[nt][i].x), scaled(qv[nt][i].y));
        s_q[warp][nt][2 * i + 1][lane] = make_uint2(scaled(qv[nt][i].z), scaled(qv[nt][i].w));
      }
    }
    far = __any_sync(0xffffffffu, far);
    auto query_of = [&](int nt, int step) { return s_q[warp][nt][step][lane]; };

    // o: dims gid-rows of a tile, query rows 2 c and 2 c + 1; nm: the lift less the running maximum
    float o[NT][MT][4], nm[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
      nm[nt][0] = nm[nt][1] = INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }
    uint32_t poison_row = 0;    // bit 2 nt + h: of row 2 c + h of tile nt
    int ek = 127, ev = 0, ev_top = 0;   // exponent bytes that keys' and values' powers are relative to (ev: none yet)
    float kp = 1.f;                      // 2^(ek - 127)
    auto scale_outputs = [&](float f) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[nt][i][k] *= f;
    };

    // The softmax step of a block or two for a tile: scores f * s in units of log2 (tokens token_of(gid) and two on, rows 2 c and 2 c + 1:
    // s[.][0], s[.][1] and s[.][2], s[.][3]) become P^T as operands, the running maximum, sum and output following.  The maximum moves
    // only when a score passes it by more than a margin.  The weights are rounded to fp16 or bf16, the values' type: their sum
    // is not.  (some_key: every row sees one of the block's keys, or one before; unit: what bf16 weights are taken times)
    auto softmax = [&](int nt, const auto& s, float f0, float f1, auto& p, bool fp16, bool some_key, float unit) {
      constexpr int kN = sizeof(s) / 16;   // blocks
      float mx[2] = {fmaxf(s[0][0], s[0][2]), fmaxf(s[0][1], s[0][3])};
#pragma unroll
      for (int x = 1; x < kN; ++x) {
        mx[0] = fmaxf(mx[0], fmaxf(s[x][0], s[x][2]));
        mx[1] = fmaxf(mx[1], fmaxf(s[x][1], s[x][3]));
      }
      mx[0] *= f0;
      mx[1] *= f1;
      if (__any_sync(0xffffffffu, mx[0] + nm[nt][0] > kLift + kMargin || mx[1] + nm[nt][1] > kLift + kMargin)) {
        float al[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = mx[h];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
          const float to = fminf(nm[nt][h], kLift - x);
          al[h] = to == nm[nt][h] ? 1.f : ex2_ftz(to - nm[nt][h]);
          nm[nt][h] = to;
          l[nt][h] *= al[h];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          o[nt][i][0] *= al[0];
          o[nt][i][1] *= al[1];
          o[nt][i][2] *= al[0];
          o[nt][i][3] *= al[1];
        }
      }
      const float n0 = some_key || nm[nt][0] < INFINITY ? nm[nt][0] : 0.f, n1 = some_key || nm[nt][1] < INFINITY ? nm[nt][1] : 0.f;
#pragma unroll
      for (int x = 0; x < kN; ++x) {
        const float w[4] = {ex2_ftz(fmaf(s[x][0], f0, n0)), ex2_ftz(fmaf(s[x][1], f1, n1)), ex2_ftz(fmaf(s[x][2], f0, n0)),
                            ex2_ftz(fmaf(s[x][3], f1, n1))};
        l[nt][0] += w[0] + w[2];
        l[nt][1] += w[1] + w[3];
        p[x][0] = transposed(fp16 ? pack_f16(w[0], w[1]) : pack_bf16(w[0] * unit, w[1] * unit));
        p[x][1] = transposed(fp16 ? pack_f16(w[2], w[3]) : pack_bf16(w[2] * unit, w[3] * unit));
      }
    };

    // ---- the cache
    // A page in the general form: the last one, or one whose powers leave the window.
    auto general = [&](int at, int place) {
      Loaded x;
      read_keys(place, x);
      read_values(place, x);
      const int b = c0 + at;
      const uint32_t ve = value_bytes(x);
      const int have = q.len - b * kTreePage;   // tokens of the page: 16 or more where it is full
      uint32_t live = 0x3Fu;   // bits 0, 1: of this lane's key rows, 2 ..: of its value rows
      if (have < kTreePage) {
        live = 0u;
#pragma unroll
        for (int n = 0; n < 2; ++n) live |= (token_of(gid) + 2 * n < have ? 1u : 0u) << n;
#pragma unroll
        for (int t = 0; t < 4; ++t) live |= (4 * c + t < have ? 4u : 0u) << t;
      }
      uint32_t kf[2], vf[2];   // factors as fp16 pairs: of a key row, of two tokens' values
      bool wide = false;       // bf16 instead
      {
        // the largest and least powers of rows within the length; blocks of the least power, 2^-127, count as nothing where their codes
        // are zeros, and are beyond any window else
        int k_most = 0, k_least = 255, v_most = 0, v_least = 255;
        bool beyond = false;   // NaN, or something in the least power: the longer products have a place for it
        auto take = [&](bool in, uint32_t field, uint32_t codes, int& most, int& least) {
          const bool something = field == 0u && (codes & 0x77777777u) != 0u;
          beyond = beyond || (in && (field == 255u || something));
          if (something) field = 1u;
          if (!in || field == 0u || field == 255u) return;
          most = max(most, static_cast<int>(field));
          least = min(least, static_cast<int>(field));
        };
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          uint32_t codes = 0;
#pragma unroll
          for (int w = 0; w < kW; ++w) codes |= x.k[n][w];
          take((live >> n) & 1u, x.ke[n], codes, k_most, k_least);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint32_t codes = 0;
#pragma unroll
          for (int w = 0; w < kVW; ++w) codes |= x.v[t][w];
          take((live >> (2 + t)) & 1u, (ve >> (8 * t)) & 255u, codes, v_most, v_least);
        }
        k_most = __reduce_max_sync(0xffffffffu, k_most);
        k_least = __reduce_min_sync(0xffffffffu, k_least);
        v_most = __reduce_max_sync(0xffffffffu, v_most);
        v_least = __reduce_min_sync(0xffffffffu, v_least);
        auto fits = [](int most, int least, int e) { return most <= e + 7 && least >= e - kBelow; };
        wide = far || __any_sync(0xffffffffu, beyond);
        if (k_most > 0 && !fits(k_most, k_least, ek)) {
          ek = min(k_least + kBelow, kTop);
          kp = power_of(ek);
          wide = wide || !fits(k_most, k_least, ek);
        }
        if (v_most > 0 && (ev == 0 || !fits(v_most, v_least, ev))) {
          // Ev goes where they fit, but not further than 2^40 below the highest that it was (the outputs have to stay
          // finite); else to where the largest does
          const int top = max(ev_top, v_most - 7);
          int to = v_least + kBelow;
          if (!fits(v_most, v_least, to) || to < top - 40) {
            to = max(top, v_most > ev + 7 ? 0 : ev);
            wide = true;
          }
          to = min(max(to, 64), kTop);   // (2^-63 and less: whatever is there loses nothing that counts)
          wide = wide || !fits(v_most, v_least, to);
          if (ev > 0) scale_outputs(power_of(min(max(127 + ev - to, 0), 254)));
          ev = to;
          ev_top = max(ev_top, ev);
        }
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const bool zero = x.ke[n] == 0u || !((live >> n) & 1u);
          kf[n] = zero || wide ? 0u : (x.ke[n] - (ek - kBelow) + 7u) * 0x04000400u;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t e = (ve >> (8 * t)) & 255u;
          const bool zero = e == 0u || !((live >> (2 + t)) & 1u);
          const uint32_t f = zero || wide ? 0u : (e - (ev - kBelow) + 7u) << 10;
          vf[t >> 1] = t & 1 ? vf[t >> 1] | f << 16 : f;
        }
      }
      // scores
      float s[NT][1][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][0][0] = s[nt][0][1] = s[nt][0][2] = s[nt][0][3] = 0.f;
      if (!wide) {
#pragma unroll
        for (int w = 0; w < kW; ++w) {
          uint32_t h0[4], h1[4];
          f16_of_e2m1(x.k[0][w], h0);
          f16_of_e2m1(x.k[1][w], h1);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            h0[i] = mul_f16x2(h0[i], kf[0]);
            h1[i] = mul_f16x2(h1[i], kf[1]);
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint2 f = query_of(nt, 2 * w + i);
              mma_f16(s[nt][0], h0[2 * i], h1[2 * i], h0[2 * i + 1], h1[2 * i + 1], f.x, f.y);
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][0][i] *= rs[nt][i & 1] * kp;
      } else {
        const float k0 = row_factor(x.ke[0]), k1 = row_factor(x.ke[1]);
#pragma unroll 1
        for (int nt = 0; nt < NT; ++nt) {
          const uint4* src = query(nt);
          float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < kW; ++w) {
            uint32_t h0[4], h1[4];
            f16_of_e2m1(x.k[0][w], h0);
            f16_of_e2m1(x.k[1][w], h1);
            const uint4 f = src ? __ldg(src + w) : make_uint4(0u, 0u, 0u, 0u);
            mma_bf16_16816(t, bf16_times(h0[0], k0, k0), bf16_times(h1[0], k1, k1), bf16_times(h0[1], k0, k0),
                           bf16_times(h1[1], k1, k1), f.x, f.y);
            mma_bf16_16816(t, bf16_times(h0[2], k0, k0), bf16_times(h1[2], k1, k1), bf16_times(h0[3], k0, k0),
                           bf16_times(h1[3], k1, k1), f.z, f.w);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int y = 0; y < NT; ++y)
              if (y == nt) s[y][0][i] = t[i] * a.scale_log2;
          }
        }
      }
      if (have < kTreePage) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((live >> (i >> 1)) & 1u)) s[nt][0][i] = -INFINITY;
      }
      uint32_t p[NT][1][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) softmax(nt, s[nt], 1.f, 1.f, p[nt], !wide, true, 1.f);
      // the weights' product with the values: words lo and hi have the even and the odd dims' codes, two tokens' side by side
#pragma unroll
      for (int w = 0; w < kVW; ++w) {
        uint32_t even[2][4], odd[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t x0 = x.v[2 * t][w], x1 = x.v[2 * t + 1][w];
          f16_of_e2m1((x0 & 0x0F0F0F0Fu) | ((x1 << 4) & 0xF0F0F0F0u), even[t]);
          f16_of_e2m1(((x0 >> 4) & 0x0F0F0F0Fu) | (x1 & 0xF0F0F0F0u), odd[t]);
        }
        if (!wide) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a0 = mul_f16x2(even[0][i], vf[0]), a1 = mul_f16x2(odd[0][i], vf[0]);
            const uint32_t a2 = mul_f16x2(even[1][i], vf[1]), a3 = mul_f16x2(odd[1][i], vf[1]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][4 * w + i], a0, a1, a2, a3, p[nt][0][0], p[nt][0][1]);
          }
        } else {
          float f[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int e = static_cast<int>((ve >> (8 * t)) & 255u);
            f[t] = !((live >> (2 + t)) & 1u) ? 0.f : e == 255 ? NAN : power_of(min(max(127 + e - ev, 0), 254));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a0 = bf16_times(even[0][i], f[0], f[1]), a1 = bf16_times(odd[0][i], f[0], f[1]);
            const uint32_t a2 = bf16_times(even[1][i], f[2], f[3]), a3 = bf16_times(odd[1][i], f[2], f[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(o[nt][4 * w + i], a0, a1, a2, a3, p[nt][0][0], p[nt][0][1]);
          }
        }
      }
    };
    poison = poison || pages < mine;
    auto scores = [&](const Loaded(&x)[P], const uint32_t(&kg)[P], float(&s)[P][NT][4]) {
      uint32_t kf[P][2];   // factors as fp16 pairs, 2^(g - 8): of a key row
#pragma unroll
      for (int y = 0; y < P; ++y) {
        kf[y][0] = __byte_perm(kg[y], 0, 0x0404) * 4u + 0x1C001C00u;
        kf[y][1] = __byte_perm(kg[y], 0, 0x1414) * 4u + 0x1C001C00u;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[y][nt][0] = s[y][nt][1] = s[y][nt][2] = s[y][nt][3] = 0.f;
      }
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        uint32_t h[P][2][4];
#pragma unroll
        for (int y = 0; y < P; ++y)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            f16_of_e2m1(x[y].k[n][w], h[y][n]);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[y][n][i] = mul_f16x2(h[y][n][i], kf[y][n]);
          }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const uint2 f = query_of(nt, 2 * w + i);
#pragma unroll
            for (int y = 0; y < P; ++y)
              mma_f16(s[y][nt], h[y][0][2 * i], h[y][1][2 * i], h[y][0][2 * i + 1], h[y][1][2 * i + 1], f.x, f.y);
          }
      }
    };
    // The weights' product with the values: words have the even or the odd dims' codes, two tokens' side by side.
    auto product = [&](int place, const uint32_t(&vg)[P], const uint32_t(&w2)[NT][P][2]) {
#pragma unroll
      for (int y = 0; y < P; ++y) {
        Loaded x;
        read_values(place + y * S::kBytes, x);
        const uint32_t vf[2] = {__byte_perm(vg[y], 0, 0x1404) * 4u + 0x1C001C00u, __byte_perm(vg[y], 0, 0x3424) * 4u + 0x1C001C00u};
#pragma unroll
        for (int w = 0; w < kVW; ++w) {
          uint32_t even[2][4], odd[2][4];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const uint32_t x0 = x.v[2 * t][w], x1 = x.v[2 * t + 1][w];
            f16_of_e2m1((x0 & 0x0F0F0F0Fu) | ((x1 << 4) & 0xF0F0F0F0u), even[t]);
            f16_of_e2m1(((x0 >> 4) & 0x0F0F0F0Fu) | (x1 & 0xF0F0F0F0u), odd[t]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a0 = mul_f16x2(even[0][i], vf[0]), a1 = mul_f16x2(odd[0][i], vf[0]);
            const uint32_t a2 = mul_f16x2(even[1][i], vf[1]), a3 = mul_f16x2(odd[1][i], vf[1]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][4 * w + i], a0, a1, a2, a3, w2[nt][y][0], w2[nt][y][1]);
          }
        }
      }
    };
    const int full = min(pages, q.len / kTreePage - c0);   // pages without places beyond the length
    int plain = 0;                                              // of these, those that the short form may take
    for (int at = 0, place = 0; at < pages; at += P) {
      copies_wait<kRing / P - 1>();
      __syncwarp();
      // powers relative to Ek and Ev, a byte each: field - (E - 8) is in 0 .. 15 for all blocks (one below it borrows)
      Loaded now[P];
      uint32_t kg[P], vg[P], out = 0;
#pragma unroll
      for (int x = 0; x < P; ++x) {   // (pages that are not there: whatever lies in the ring)
        read_keys(place + x * S::kBytes, now[x]);
        kg[x] = (now[x].ke[0] | now[x].ke[1] << 8) - static_cast<uint32_t>(ek - kBelow) * 0x0101u;
        vg[x] = value_bytes(now[x]) - static_cast<uint32_t>(ev - kBelow) * 0x01010101u;
        out |= (kg[x] & ~0x0F0Fu) | (vg[x] & 0xF0F0F0F0u);
      }
      if (__any_sync(0xffffffffu, out != 0u) || at + P > plain) {
#pragma unroll 1
        for (int x = 0; x < min(pages - at, P); ++x) general(at + x, place + x * S::kBytes);
        plain = ev != 0 && !far ? full : 0;
      } else {
        float s[P][NT][4];
        scores(now, kg, s);
        uint32_t p[NT][P][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float y[P][4];
#pragma unroll
          for (int x = 0; x < P; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[x][i] = s[x][nt][i];
          softmax(nt, y, rs[nt][0] * kp, rs[nt][1] * kp, p[nt], true, true, 1.f);
        }
        product(place, vg, p);
      }
      __syncwarp();   // the places have been read
      fetch(at + kRing, ring + place);
      place = place == (kRing - P) * S::kBytes ? 0 : place + P * S::kBytes;
    }
    copies_wait<0>();

    // ---- drafted tokens: bf16 rows of their own tensors, whatever the cache holds
    if (ev == 0) ev = 127;   // (nothing so far)
    for (int b = c0 + mine; b < c1; ++b) {
      const int j0 = (b - q.cached_blocks) * kTreePage, have = q.drafts - j0;
      const __nv_bfloat16* kd = static_cast<const __nv_bfloat16*>(a.t.k) + (q.start + static_cast<int64_t>(j0)) * a.t.k_token + g * a.t.k_head;
      const __nv_bfloat16* vd = static_cast<const __nv_bfloat16*>(a.t.v) + (q.start + static_cast<int64_t>(j0)) * a.t.v_token + g * a.t.v_head;
      float s[NT][1][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][0][0] = s[nt][0][1] = s[nt][0][2] = s[nt][0][3] = 0.f;
#pragma unroll 1
      for (int w = 0; w < HD / 32; ++w) {   // two steps
        uint4 x[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int t = token_of(gid) + 2 * n;
          x[n] = t < have ? __ldg(reinterpret_cast<const uint4*>(kd + t * a.t.k_token + c * (HD / 4)) + w) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4* src = query(nt);
          const uint4 f = src ? __ldg(src + w) : make_uint4(0u, 0u, 0u, 0u);
          mma_bf16_16816(s[nt][0], x[0].x, x[1].x, x[0].y, x[1].y, f.x, f.y);
          mma_bf16_16816(s[nt][0], x[0].z, x[1].z, x[0].w, x[1].w, f.z, f.w);
        }
      }
      constexpr int kD = HD / 64;   // 16-byte pieces of a lane's dims of a value row
      uint4 v[4][kD];
      uint32_t bad = 0;   // tokens whose value row is not finite
      uint32_t most = 0;  // the others' largest magnitudes
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int tok = 4 * c + t;
        uint32_t magnitude = 0;
#pragma unroll
        for (int d = 0; d < kD; ++d) {
          v[t][d] = tok < have ? __ldg(reinterpret_cast<const uint4*>(vd + tok * a.t.v_token + gid * (HD / 8)) + d) : make_uint4(0u, 0u, 0u, 0u);
          magnitude = max_u16x2(magnitude, magnitude2(v[t][d]));
        }
        const uint32_t who = __ballot_sync(0xffffffffu, from(magnitude, 255));
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (who & (0x11111111u << x)) bad |= 1u << (4 * x + t);
        if ((bad >> tok) & 1u) {   // a weight of zero must leave no trace of it: rows that see it are marked instead
#pragma unroll
          for (int d = 0; d < kD; ++d) v[t][d] = make_uint4(0u, 0u, 0u, 0u);
          magnitude = 0;
        }
        most = max_u16x2(most, magnitude);
      }
      // Outputs are kept in units of 1 at least, for drafted values times a larger power might not be finite.  Weights are 2^15 at
      // most and may be many: beside values of 2^88 and more the units are 2^40 at least, so that the sums stay finite (an output
      // below 2^-98 loses bits beside such values).  Up to 2^40 of a unit goes to the weights, whose least that counts is
      // far above bf16's least, the rest to the products.
      const int least = __any_sync(0xffffffffu, from(most, 127 + 88)) ? 127 + 40 : 127;
      if (ev < least) {
        scale_outputs(power_of(127 + ev - least));
        ev = least;
      }
      const float unit = power_of(max(254 - ev, 127 - 40)), rest = power_of(min(254 - ev + 40, 127));
      uint32_t p[NT][1][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = row0 + 8 * nt + 2 * c + h;
          const uint32_t sees = r < rows ? tree_sees16(a, q, tree_token(a, r), j0) : 0u;
          if (sees & bad) poison_row |= 1u << (2 * nt + h);
#pragma unroll
          for (int n = 0; n < 2; ++n)
            s[nt][0][2 * n + h] = (sees >> (token_of(gid) + 2 * n)) & 1u ? s[nt][0][2 * n + h] * a.scale_log2 : -INFINITY;
        }
        softmax(nt, s[nt], 1.f, 1.f, p[nt], false, false, unit);
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int d = i / 4;
        auto word = [&](int t) { return i % 4 == 0 ? v[t][d].x : i % 4 == 1 ? v[t][d].y : i % 4 == 2 ? v[t][d].z : v[t][d].w; };
        uint32_t x[4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          x[2 * t] = __byte_perm(word(2 * t), word(2 * t + 1), 0x5410);
          x[2 * t + 1] = __byte_perm(word(2 * t), word(2 * t + 1), 0x7632);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float t[4] = {0.f, 0.f, 0.f, 0.f};
          mma_bf16_16816(t, x[0], x[1], x[2], x[3], p[nt][0][0], p[nt][0][1]);
#pragma unroll
          for (int k = 0; k < 4; ++k) o[nt][i][k] += t[k] * rest;
        }
      }
    }

    // ---- the part's end
    // What a part leaves is its own mean, in the values' own scale, with the sum of its weights beside it: the sum of weights
    // times values may be beyond fp32 where the mean is not.
    const bool lost = __any_sync(0xffffffffu, poison);
    float mean[NT][2];   // what makes a mean of an output
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = l[nt][h];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lost || (poison_row >> (2 * nt + h)) & 1u) sum = NAN;
        l[nt][h] = sum;
        mean[nt][h] = sum == 0.f ? 0.f : __fdividef(power_of(ev), sum);   // a row that saw nothing: zeros; NaN stays
      }
    if constexpr (WHOLE) {   // the warps' states meet, 8 rows at a time, in their rings
      constexpr int kOutRow = HD + 4, kPer = 8 * HD / kThreads;   // kPer: outputs of a thread, part of one row
      auto out_of = [&](int w) { return reinterpret_cast<float*>(s_ring + w * (kRing * S::kBytes)); };
      static_assert(8 * kOutRow * 4 <= kRing * S::kBytes, "a warp's rows fit its ring");
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (row0 + 8 * nt >= rows) break;   // (the same for all threads)
        if (nt > 0) __syncthreads();        // the last 8 rows have been read
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float f = mean[nt][h];
          if (gid == 0) s_ml[warp][2 * c + h] = make_float2(-nm[nt][h], l[nt][h]);
#pragma unroll
          for (int i = 0; i < MT; ++i)   // dims 2 i and 2 i + 1 of this lane's HD / 8
            *reinterpret_cast<float2*>(out_of(warp) + (2 * c + h) * kOutRow + gid * (HD / 8) + 2 * i) = make_float2(o[nt][i][h] * f, o[nt][i][2 + h] * f);
        }
        __syncthreads();
        const int r = threadIdx.x / 16, d0 = threadIdx.x % 16 * kPer, out_r = row0 + 8 * nt + r;
        float top = -INFINITY, sum = 0.f, acc[kPer];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, part_top(s_ml[w][r]));
#pragma unroll
        for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = part_weight(s_ml[w][r], top);
          sum += f;
#pragma unroll
          for (int i = 0; i < kPer; ++i) acc[i] += out_of(w)[r * kOutRow + d0 + i] * f;
        }
        if (out_r >= rows) continue;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that saw nothing: zeros; NaN stays
        const int tok = tree_token(a, out_r);
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.t.out) + (q.start + static_cast<int64_t>(tok)) * a.t.out_token +
                             (g * a.group + out_r - tok * a.group) * a.t.out_head + d0;
        uint32_t w[kPer / 2];
#pragma unroll
        for (int i = 0; i < kPer / 2; ++i) w[i] = pack_bf16(acc[2 * i] * inv, acc[2 * i + 1] * inv);
        if constexpr (kPer == 8)
          *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        else
          *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
      }
      __syncthreads();   // the rings are free for the next part
      continue;
    }
    if constexpr (!WHOLE) {
      const bool whole = part.whole();
      // partial results: [row][dim]
      const int64_t slot = me == shares.owner(part.place(0)) ? 2 * me + 1 : 2 * me;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int slot_row = 8 * nt + 2 * c + h, r = row0 + slot_row;
          if (r >= rows) continue;
          float y[2 * MT];   // this lane's HD / 8 dims
          const float f = mean[nt][h];
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            y[2 * i] = o[nt][i][h] * f;
            y[2 * i + 1] = o[nt][i][2 + h] * f;
          }
          if (whole) {
            const int tok = tree_token(a, r);
            __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.t.out) + (q.start + static_cast<int64_t>(tok)) * a.t.out_token +
                                 (g * a.group + r - tok * a.group) * a.t.out_head + gid * (HD / 8);
#pragma unroll
            for (int i = 0; i < 2 * MT; i += 8)
              *reinterpret_cast<uint4*>(dst + i) = make_uint4(pack_bf16(y[i], y[i + 1]), pack_bf16(y[i + 2], y[i + 3]),
                                                              pack_bf16(y[i + 4], y[i + 5]), pack_bf16(y[i + 6], y[i + 7]));
          } else {
            float* dst = a.part_o + (slot * G::kSlotRows + slot_row) * HD + gid * (HD / 8);
#pragma unroll
            for (int i = 0; i < 2 * MT; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
            if (gid == 0) a.part_ml[slot * G::kSlotRows + slot_row] = make_float2(-nm[nt][h], l[nt][h]);
          }
        }
      }
    }
    __syncwarp();
  }
}

// Joins the partial results of pairs that several warps shared, eight rows and 64 dims of a pair a CTA: launched beside the
// attention kernel's end, it waits for it; each of W warps takes every W-th part, in order, and their states meet in shared
// memory, so the result does not depend on who was last.  A lane has four times four dims of a row, 16 apart.
//
// What it costs is latencies: 5 us of the 48 of 64 ragged sequences of 4 heads (256 pairs of some eight parts), of which 1.4 are a
// launch's and 2 the line's.  Eight warps, or sixteen where so few CTAs leave SMs idle (that call / one sequence of 32,768 tokens with 64
// parts a pair: eight 47.7 / 26.2, sixteen 50.5 / 24.4; four with 32 dims and four parts ahead 48.6 / 27.4; eight with 128 dims 48.2 / 29.5).
// Weighing means instead of sums by their own reciprocals, part after part, 0.5 more than by powers of two (part_top).
constexpr int kJoinDims = 64, kJoinFew = 128;
template <int HD, int NT, int W>
__global__ void __launch_bounds__(32 * W) tree_e2m1_join_kernel(const __grid_constant__ TreeLaunch a, int groups) {
  using G = TreeE2m1<NT>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, d0 = blockIdx.y * kJoinDims + (lane & 3) * 4;
  const int group = blockIdx.x % groups, head = blockIdx.x / groups, g = head % a.n_kv, s = head / a.n_kv;
  const TreeSeq q = tree_seq<G::ROWS, G::BLOCK>(a, s);
  const int rows = q.drafts * a.group, row = 8 * group + r, tp = 8 * group / G::kSlotRows, slot_row = row - tp * G::kSlotRows;
  grid_dep_wait();   // no launch of this kernel ends before the attention kernel
  const int32_t off = __ldcg(a.line + s), total = __ldcg(a.line + a.n_seqs), ctas = __ldcg(a.line + a.n_seqs + 1);
  if (8 * group >= rows) return;
  const TreeShares shares(total, ctas, 1);
  const int32_t first = off + (q.blocks + G::LEAD) * (g * q.tiles + tp) + G::LEAD;   // (a place is a block: weights of 1)
  const int i0 = shares.owner(first), i1 = shares.owner(first + q.blocks - 1);
  if (i0 == i1) return;   // whole: written by its warp
  __shared__ float s_o[W][32][17];
  __shared__ float2 s_ml[W][8];
  float o[16] = {}, best = -INFINITY, sum = 0.f;
#pragma unroll 1
  for (int part = i0 + warp; part <= i1; part += W) {
    const int64_t at = (part == i0 ? 2 * i0 + 1 : 2 * part) * static_cast<int64_t>(G::kSlotRows) + slot_row;
    const float2 ml = __ldcg(a.part_ml + at);
    float4 v[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) v[d] = __ldcg(reinterpret_cast<const float4*>(a.part_o + at * HD + d0 + 16 * d));
    const float now = fmaxf(best, part_top(ml));   // -infinity: nothing seen so far (a sum of zero, or NaN)
    const float f = best == -INFINITY ? 0.f : ex2_ftz(best - now), e = part_weight(ml, now);
    best = now;
    sum = sum * f + e;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      o[4 * d] = o[4 * d] * f + v[d].x * e;
      o[4 * d + 1] = o[4 * d + 1] * f + v[d].y * e;
      o[4 * d + 2] = o[4 * d + 2] * f + v[d].z * e;
      o[4 * d + 3] = o[4 * d + 3] * f + v[d].w * e;
    }
  }
#pragma unroll
  for (int d = 0; d < 16; ++d) s_o[warp][lane][d] = o[d];
  if ((lane & 3) == 0) s_ml[warp][r] = make_float2(best, sum);
  __syncthreads();
  if (warp >= 4 || row >= rows) return;   // a warp for each of the lanes' fours
  float top = -INFINITY, all = 0.f, y[4] = {};
#pragma unroll
  for (int w = 0; w < W; ++w) top = fmaxf(top, s_ml[w][r].x);
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float f = s_ml[w][r].x == -INFINITY ? 0.f : ex2_ftz(s_ml[w][r].x - top);   // (NaN sums stay NaN)
    all += s_ml[w][r].y * f;
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] += s_o[w][lane][4 * warp + d] * f;
  }
  const float inv = all == 0.f ? 0.f : 1.f / all;
  const int tok = tree_token(a, row);
  __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.t.out) + (q.start + static_cast<int64_t>(tok)) * a.t.out_token +
                       (g * a.group + row - tok * a.group) * a.t.out_head + d0 + 16 * warp;
  *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv));
}

template <int HD, int NT>
cudaError_t launch_join(const TreeLaunch& a, cudaStream_t stream) {
  const int groups = (a.t.max_drafts * a.group + 7) / 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(static_cast<int64_t>(a.n_seqs) * a.n_kv * groups), HD / kJoinDims);
  const bool few = int64_t{cfg.gridDim.x} * cfg.gridDim.y <= kJoinFew;
  cfg.blockDim = dim3(few ? 512 : 256);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, few ? tree_e2m1_join_kernel<HD, NT, 16> : tree_e2m1_join_kernel<HD, NT, 8>, a, groups);
}

template <int HD, int NT, bool WHOLE>
cudaError_t launch(const TreeLaunch& a, int ctas, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  // (beyond 48 KB a launch has to ask; a decoding step's are within, and it costs the host a microsecond)
  constexpr size_t kStatic = 4 * (kTreeSeqs + 1) + 4 * kWarps + sizeof(uint2) * kWarps * (NT * (HD / 16) * 32 + 8) + 64;
  if constexpr (kStatic + ring_bytes<HD>() > 48 * 1024)
    e = cudaFuncSetAttribute(tree_e2m1_kernel<HD, NT, WHOLE>, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes<HD>());
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = ring_bytes<HD>();
  cfg.stream = stream;
  e = cudaLaunchKernelEx(&cfg, tree_e2m1_kernel<HD, NT, WHOLE>, a);
  return e == cudaSuccess && !WHOLE && a.n_seqs > 0 ? launch_join<HD, NT>(a, stream) : e;
}
template <int HD, int NT>
cudaError_t launch(const TreeLaunch& a, int ctas, cudaStream_t stream) {
  return a.whole ? launch<HD, NT, true>(a, ctas, stream) : launch<HD, NT, false>(a, ctas, stream);
}

}  // namespace

cudaError_t launch_tree_e2m1(const TreeLaunch& a, const kvprm_cache& c, int tiles, int ctas, cudaStream_t stream) {
  const bool wide = c.head_dim == 128;
  if (tiles == 1) return wide ? launch<128, 1>(a, ctas, stream) : launch<64, 1>(a, ctas, stream);
  if (tiles == 2) return wide ? launch<128, 2>(a, ctas, stream) : launch<64, 2>(a, ctas, stream);
  return wide ? launch<128, 4>(a, ctas, stream) : launch<64, 4>(a, ctas, stream);
}

}  // namespace kvprm
