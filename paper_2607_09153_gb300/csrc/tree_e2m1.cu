// Attention of drafted tokens over 4-bit pages (e2m1 codes, a power of two for each 32 elements): up to 32 query rows (row =
// drafted token and head of the kv head's group) a tile, by warp-level matrix instructions on fragments that are loaded
// straight from the pages.
//
// The products are the transposed ones, S^T = K Q^T and O^T = V^T P^T: the cache's rows fill the 16 rows of an instruction
// and the queries its 8 columns, so a plain decoding step (up to 8 query heads on a kv head) takes half the instructions
// that tiles of 16 query rows take.  A lane's 16 bytes of a key row are one block of 32 elements: it converts them (one
// instruction for two codes, to fp16), multiplies them by the block's power of two, and has the operands of eight steps;
// dimensions run in any order as long as Q's follow.  Of the values a lane has the same 16 dimensions of four tokens: the
// nibbles of two tokens are put side by side, so that one conversion gives an operand's pair.  S^T's columns become P^T's
// by one 8 x 8 transposition in registers.
//
// What fp16 lacks in range is kept beside it as powers of two.  A query row is scaled to a largest magnitude of 1 to 2 (exact
// but for elements 2^-14 of that and smaller, which lose what is below 2^-25 of it).  A page's key blocks are taken
// relative to a power Ek that its scores are multiplied by in fp32, the values' relative to a power Ev that the outputs are kept
// relative to: blocks from 2^-8 to 2^7 of it are exact.  A page that leaves that window moves Ek or Ev; one whose own
// blocks are further apart takes its products in bf16 instead, whose range is fp32's.  Weights are kept times 2^12, so
// that fp16's steps end at 2^-36 of a full weight's.
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

__device__ __forceinline__ uint4 ldg16(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}
__device__ __forceinline__ uint2 ldg8(const void* p) {
  uint2 r;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint32_t ldg4(const void* p) {
  uint32_t r;
  asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(r) : "l"(p));
  return r;
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
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}
// Two codes' fp16 times factors, as bf16 (the longer form).
__device__ __forceinline__ uint32_t bf16_times(uint32_t h, float lo, float hi) {
  const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return pack_bf16(v.x * lo, v.y * hi);
}
// The token of a page that row r of S^T, and index r of P V's sums, stand for: a lane's four values' rows are neighbours.
__device__ __forceinline__ int token_of(int r) { return 4 * ((r & 7) >> 1) + (r & 1) + ((r >> 3) << 1); }

// NT: tiles of 8 query rows.
template <int HD, int NT>
__global__ void __launch_bounds__(kThreads, tree_e2m1_per_sm(NT)) tree_e2m1_kernel(const __grid_constant__ TreeLaunch a) {
  using G = TreeRows<NT <= 2 ? 1 : 2>;
  constexpr int KS = HD / 16;            // 16-dim steps of q . k
  constexpr int MT = HD / 16;            // 16-dim tiles of the output
  constexpr int kW = HD / 32;            // a lane's words of a key row, of eight codes
  constexpr int kVW = HD / 64;           // of each of its four value rows
  constexpr int kRowBytes = HD / 2, kBlocks = HD / 32;
  __shared__ int32_t s_off[kTreeSeqs + 1];
  __shared__ int32_t s_sum[kWarps];
  __shared__ union {
    uint2 q[NT][KS][32];              // the scaled queries' fragments, by lane
    float o[kWarps][8][HD + 4];       // at a part's end, the warps' outputs
  } sh;
  __shared__ float s_m[kWarps][8], s_l[kWarps][8];
  grid_dep_launch();
  tree_line<G, kThreads, HD>(a, s_off, s_sum);
  const int32_t total = s_off[a.n_seqs];
  if (total == 0) return;
  const TreeShares shares(total, gridDim.x, a.weight_full);
  const int me = blockIdx.x;
  tree_leave_line(a, s_off, shares.ctas);
  if (me >= shares.ctas) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, c = lane & 3;
  const int64_t head_bytes = kTreePage * kRowBytes, page_bytes = 2 * a.n_kv * head_bytes;
  constexpr int kHeadExp = kTreePage * kBlocks;
  const int64_t page_exp = 2 * static_cast<int64_t>(a.n_kv) * kHeadExp;
  int32_t u = shares.begin(me);
  const int32_t u_end = shares.begin(me + 1);
  int s_at = tree_find(s_off, a.n_seqs, u);
  TreePart part;
  while (tree_next<G>(a, s_off, u, u_end, s_at, part)) {
    const TreeSeq& q = part.q;
    const int g = part.g, row0 = part.tp * G::kSlotRows, rows = q.drafts * a.group;
    const int32_t* table = a.t.block_table + static_cast<int64_t>(a.seq0 + s_at) * a.t.max_blocks;
    // this lane's bytes of a page: piece c of key row token_of(gid) (the other two rows on), dims of gid of value rows 4 c ..
    const uint8_t* keys = a.pages + g * head_bytes + token_of(gid) * kRowBytes + c * (kRowBytes / 4);
    const uint8_t* values = a.pages + (a.n_kv + g) * head_bytes + 4 * c * kRowBytes + gid * (kRowBytes / 8);
    const uint8_t* key_exp = a.exponents + g * kHeadExp + token_of(gid) * kBlocks + c * kBlocks / 4;
    const uint8_t* value_exp = a.exponents + (a.n_kv + g) * kHeadExp + 4 * c * kBlocks;
    // the query rows' elements (HD / 4) c .. of row gid of tile nt
    auto query = [&](int nt) -> const uint4* {
      const int r = row0 + 8 * nt + gid;
      if (r >= rows) return nullptr;
      const int tok = tree_token(a, r);
      return reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.t.q) + (q.start + static_cast<int64_t>(tok)) * a.t.q_token +
                                            (g * a.group + r - tok * a.group) * a.t.q_head + c * (HD / 4));
    };

    // ---- the queries, scaled: warp w makes tiles w, w + 4
    float rs[NT][2];   // of rows 2 c and 2 c + 1: the row's power of two times the scores' scale
    __syncthreads();   // the last part's have been read
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint4* src = query(nt);
      uint4 v[HD / 32];
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        v[i] = src ? __ldg(src + i) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) most = fmaxf(most, fmaxf(fabsf(lo_bf16(w[k])), fabsf(hi_bf16(w[k]))));
      }
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      int e = static_cast<int>(__float_as_uint(most) >> 23);   // (infinite or all zero: any scale does)
      e = e < 1 || e > 253 ? 127 : e;
      rs[nt][0] = __shfl_sync(0xffffffffu, power_of(e), 8 * c) * a.scale_log2;
      rs[nt][1] = __shfl_sync(0xffffffffu, power_of(e), 8 * c + 4) * a.scale_log2;
      if ((nt & (kWarps - 1)) != warp) continue;
      const float up = power_of(254 - e);
      auto scaled = [&](uint32_t x) { return pack_f16(lo_bf16(x) * up, hi_bf16(x) * up); };
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        sh.q[nt][2 * i][lane] = make_uint2(scaled(v[i].x), scaled(v[i].y));
        sh.q[nt][2 * i + 1][lane] = make_uint2(scaled(v[i].z), scaled(v[i].w));
      }
    }
    __syncthreads();

    float o[NT][MT][4], m[NT][2], l[NT][2];   // o: dims gid-rows of a tile, query rows 2 c and 2 c + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }
    bool poison = q.bad;        // of all rows of the sequence
    uint32_t poison_row = 0;    // bit 2 nt + h: of row 2 c + h of tile nt
    int ek = 127, ev = -64, ev_top = 0;   // exponent bytes that keys' and values' powers are relative to (ev: none yet)
    auto scale_outputs = [&](float f) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[nt][i][k] *= f;
    };

    // One block's softmax step for a tile: scores s in units of log2 (tokens token_of(gid) and two on, rows 2 c and 2 c + 1:
    // s[0], s[1] and s[2], s[3]) become P^T as an operand, the running maximum, sum and output following.  The maximum moves
    // only when a score passes it by more than a margin.  The weights are rounded to fp16 or bf16, the values' type: their sum
    // is not.
    auto softmax = [&](int nt, const float(&s)[4], uint32_t(&p)[2], bool fp16) {
      const float mx[2] = {fmaxf(s[0], s[2]), fmaxf(s[1], s[3])};
      if (__any_sync(0xffffffffu, mx[0] > m[nt][0] + kMargin || mx[1] > m[nt][1] + kMargin)) {
        float al[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = mx[h];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
          x = fmaxf(x, m[nt][h]);
          al[h] = x == m[nt][h] ? 1.f : ex2_ftz(m[nt][h] - x);
          m[nt][h] = x;
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
      float w[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float nm = m[nt][h] == -INFINITY ? kLift : kLift - m[nt][h];   // nothing seen yet: every score is -infinity
        w[h] = ex2_ftz(s[h] + nm);
        w[2 + h] = ex2_ftz(s[2 + h] + nm);
        l[nt][h] += w[h] + w[2 + h];
      }
      p[0] = transposed(fp16 ? pack_f16(w[0], w[1]) : pack_bf16(w[0], w[1]));
      p[1] = transposed(fp16 ? pack_f16(w[2], w[3]) : pack_bf16(w[2], w[3]));
    };

    const int c_end = min(part.c1, q.cached_blocks);
    auto page_of = [&](int b) { return b < c_end ? __ldg(table + b) : 0; };
    auto in_cache = [&](int32_t page) { return page >= 0 && page < a.n_pages; };
    struct Loaded {
      uint32_t k[2][kW], v[4][kVW];
      uint32_t ke[2], ve[kBlocks];   // ve: the blocks of four tokens' values
    };
    auto load = [&](int32_t page, Loaded& x) {
      const int64_t at = in_cache(page) ? page : 0;
      const uint8_t* k = keys + at * page_bytes;
      const uint8_t* v = values + at * page_bytes;
      const uint8_t* ke = key_exp + at * page_exp;
      const uint8_t* ve = value_exp + at * page_exp;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if constexpr (HD == 128) {
          const uint4 r = ldg16(k + 2 * n * kRowBytes);
          x.k[n][0] = r.x, x.k[n][1] = r.y, x.k[n][2] = r.z, x.k[n][3] = r.w;
        } else {
          const uint2 r = ldg8(k + 2 * n * kRowBytes);
          x.k[n][0] = r.x, x.k[n][1] = r.y;
        }
        x.ke[n] = __ldg(ke + 2 * n * kBlocks);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (HD == 128) {
          const uint2 r = ldg8(v + t * kRowBytes);
          x.v[t][0] = r.x, x.v[t][1] = r.y;
        } else {
          x.v[t][0] = ldg4(v + t * kRowBytes);
        }
      }
      if constexpr (HD == 128) {
        const uint4 r = __ldg(reinterpret_cast<const uint4*>(ve));
        x.ve[0] = r.x, x.ve[1] = r.y, x.ve[2] = r.z, x.ve[3] = r.w;
      } else {
        const uint2 r = __ldg(reinterpret_cast<const uint2*>(ve));
        x.ve[0] = r.x, x.ve[1] = r.y;
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

    // ---- the cache: pages b, b + 4, ..; the next page's bytes are on their way while this one's are used
    int b = part.c0 + warp;
    int32_t page = page_of(b), next = page_of(b + kWarps);
    Loaded now;
    const bool some = a.n_pages > 0;
    if (b < c_end && some) load(page, now);
    for (; b < c_end; b += kWarps) {
      if (!some) {   // an empty pool: every page is outside it
        poison = true;
        continue;
      }
      const int32_t after = page_of(b + 2 * kWarps);
      const int have = q.len - b * kTreePage;   // tokens of the page: 16 or more where it is full
      poison = poison || !in_cache(page);
      Loaded x = now;
      if (b + kWarps < c_end) load(next, now);
      uint32_t ve = value_bytes(x);
      uint32_t live = 0x3Fu;   // bits 0, 1: of this lane's key rows, 2 ..: of its value rows
      if (have < kTreePage) {
        live = 0u;
#pragma unroll
        for (int n = 0; n < 2; ++n) live |= (token_of(gid) + 2 * n < have ? 1u : 0u) << n;
#pragma unroll
        for (int t = 0; t < 4; ++t) live |= (4 * c + t < have ? 4u : 0u) << t;
      }
      // Powers relative to Ek and Ev: field - (E - 8) is in 0 .. 15 for all blocks, or the longer form looks what to do.
      uint32_t kg[2], vg[4];
#pragma unroll
      for (int n = 0; n < 2; ++n) kg[n] = x.ke[n] - (ek - kBelow);
#pragma unroll
      for (int t = 0; t < 4; ++t) vg[t] = ((ve >> (8 * t)) & 255u) - (ev - kBelow);
      uint32_t kf[2], vf[2];   // factors as fp16 pairs: of a key row, of two tokens' values
      bool wide = false;
      if (!__any_sync(0xffffffffu, live != 0x3Fu || ((kg[0] | kg[1] | vg[0] | vg[1] | vg[2] | vg[3]) & ~15u) != 0u)) {
#pragma unroll
        for (int n = 0; n < 2; ++n) kf[n] = (kg[n] + 7u) * 0x04000400u;   // 2^(g - 8) in both halves
#pragma unroll
        for (int t = 0; t < 2; ++t) vf[t] = (vg[2 * t] + 7u) * 0x0400u + (vg[2 * t + 1] + 7u) * 0x04000000u;
      } else {
        // the largest and least powers of rows within the length; blocks of the least power, 2^-127, count as nothing
        int k_most = 0, k_least = 255, v_most = 0, v_least = 255;
        bool nan = false;
        auto take = [&](bool in, uint32_t field, int& most, int& least) {
          nan = nan || (in && field == 255u);
          if (!in || field == 0u || field == 255u) return;
          most = max(most, static_cast<int>(field));
          least = min(least, static_cast<int>(field));
        };
#pragma unroll
        for (int n = 0; n < 2; ++n) take((live >> n) & 1u, x.ke[n], k_most, k_least);
#pragma unroll
        for (int t = 0; t < 4; ++t) take((live >> (2 + t)) & 1u, (ve >> (8 * t)) & 255u, v_most, v_least);
        k_most = __reduce_max_sync(0xffffffffu, k_most);
        k_least = __reduce_min_sync(0xffffffffu, k_least);
        v_most = __reduce_max_sync(0xffffffffu, v_most);
        v_least = __reduce_min_sync(0xffffffffu, v_least);
        auto fits = [](int most, int least, int e) { return most <= e + 7 && least >= e - kBelow; };
        wide = __any_sync(0xffffffffu, nan);   // (the longer products have a place for it)
        if (k_most > 0 && !fits(k_most, k_least, ek)) {
          ek = k_least + kBelow;
          wide = wide || !fits(k_most, k_least, ek);
        }
        if (v_most > 0 && !fits(v_most, v_least, ev)) {
          // Ev goes where they fit, but not further than 2^40 below the highest that it was (the outputs have to stay
          // finite); else to where the largest does
          const int top = max(ev_top, v_most - 7);
          int to = v_least + kBelow;
          if (!fits(v_most, v_least, to) || to < top - 40) {
            to = max(top, v_most > ev + 7 ? 0 : ev);
            wide = true;
          }
          to = max(to, 64);   // (2^-63 and less: whatever is there loses nothing that counts)
          wide = wide || !fits(v_most, v_least, to);
          if (ev >= 0) scale_outputs(power_of(min(max(127 + ev - to, 0), 254)));
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
      float s[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
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
              const uint2 f = sh.q[nt][2 * w + i][lane];
              mma_f16(s[nt], h0[2 * i], h1[2 * i], h0[2 * i + 1], h1[2 * i + 1], f.x, f.y);
            }
        }
        const float kp = power_of(min(max(ek, 1), 254));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][i] *= rs[nt][i & 1] * kp;
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
              if (y == nt) s[y][i] = t[i] * a.scale_log2;
          }
        }
      }
      if (have < kTreePage) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((live >> (i >> 1)) & 1u)) s[nt][i] = -INFINITY;
      }
      uint32_t p[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) softmax(nt, s[nt], p[nt], !wide);
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
            for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][4 * w + i], a0, a1, a2, a3, p[nt][0], p[nt][1]);
          }
        } else {
          float f[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int e = static_cast<int>((ve >> (8 * t)) & 255u);
            f[t] = !((live >> (2 + t)) & 1u) ? 0.f : e == 255 ? NAN : power_of(min(max(e == 0 ? 0 : 127 + e - ev, 0), 254));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a0 = bf16_times(even[0][i], f[0], f[1]), a1 = bf16_times(odd[0][i], f[0], f[1]);
            const uint32_t a2 = bf16_times(even[1][i], f[2], f[3]), a3 = bf16_times(odd[1][i], f[2], f[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(o[nt][4 * w + i], a0, a1, a2, a3, p[nt][0], p[nt][1]);
          }
        }
      }
      page = next;
      next = after;
    }

    // ---- drafted tokens: bf16 rows of their own tensors, whatever the cache holds (b is the warp's next block after the cache)
    if (ev < 0) ev = 127;
    const float rel = power_of(254 - ev);   // what the outputs are kept in, over the values' own
    for (; b < part.c1; b += kWarps) {
      const int j0 = (b - q.cached_blocks) * kTreePage, have = q.drafts - j0;
      const __nv_bfloat16* kd = static_cast<const __nv_bfloat16*>(a.t.k) + (q.start + static_cast<int64_t>(j0)) * a.t.k_token + g * a.t.k_head;
      const __nv_bfloat16* vd = static_cast<const __nv_bfloat16*>(a.t.v) + (q.start + static_cast<int64_t>(j0)) * a.t.v_token + g * a.t.v_head;
      float s[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
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
          mma_bf16_16816(s[nt], x[0].x, x[1].x, x[0].y, x[1].y, f.x, f.y);
          mma_bf16_16816(s[nt], x[0].z, x[1].z, x[0].w, x[1].w, f.z, f.w);
        }
      }
      constexpr int kD = HD / 64;   // 16-byte pieces of a lane's dims of a value row
      uint4 v[4][kD];
      uint32_t bad = 0;   // tokens whose value row is not finite
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int tok = 4 * c + t;
        bool off = false;
#pragma unroll
        for (int d = 0; d < kD; ++d) {
          v[t][d] = tok < have ? __ldg(reinterpret_cast<const uint4*>(vd + tok * a.t.v_token + gid * (HD / 8)) + d) : make_uint4(0u, 0u, 0u, 0u);
          off = off || not_finite2(v[t][d].x) || not_finite2(v[t][d].y) || not_finite2(v[t][d].z) || not_finite2(v[t][d].w);
        }
        const uint32_t who = __ballot_sync(0xffffffffu, off);
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (who & (0x11111111u << x)) bad |= 1u << (4 * x + t);
        if ((bad >> tok) & 1u) {   // a weight of zero must leave no trace of it: rows that see it are marked instead
#pragma unroll
          for (int d = 0; d < kD; ++d) v[t][d] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      uint32_t p[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = row0 + 8 * nt + 2 * c + h;
          const uint32_t sees = r < rows ? tree_sees16(a, q, tree_token(a, r), j0) : 0u;
          if (sees & bad) poison_row |= 1u << (2 * nt + h);
#pragma unroll
          for (int n = 0; n < 2; ++n)
            s[nt][2 * n + h] = (sees >> (token_of(gid) + 2 * n)) & 1u ? s[nt][2 * n + h] * a.scale_log2 : -INFINITY;
        }
        softmax(nt, s[nt], p[nt], false);
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
          mma_bf16_16816(t, x[0], x[1], x[2], x[3], p[nt][0], p[nt][1]);
#pragma unroll
          for (int k = 0; k < 4; ++k) o[nt][i][k] += t[k] * rel;
        }
      }
    }

    // ---- the part's end: the four warps' states meet, 8 rows at a time
    const float down = power_of(ev);   // 1 / rel
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (row0 + 8 * nt >= rows) break;   // (the same for all threads)
      __syncthreads();   // the queries (or the last 8 rows) have been read
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = l[nt][h];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (poison || (poison_row >> (2 * nt + h)) & 1u) sum = NAN;
        if (gid == 0) {
          s_m[warp][2 * c + h] = m[nt][h];
          s_l[warp][2 * c + h] = sum;
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i)   // dims 2 i and 2 i + 1 of this lane's HD / 8
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float2*>(&sh.o[warp][2 * c + h][gid * (HD / 8) + 2 * i]) = make_float2(o[nt][i][h] * down, o[nt][i][2 + h] * down);
      __syncthreads();
      constexpr int kPer = 8 * HD / kThreads;   // outputs of a thread: part of one row
      const int r = threadIdx.x / 16, d0 = threadIdx.x % 16 * kPer;
      float top = -INFINITY, sum = 0.f, acc[kPer];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][r]);
#pragma unroll
      for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = s_m[w][r] == -INFINITY ? 0.f : ex2_ftz(s_m[w][r] - top);   // (NaN sums stay NaN)
        sum += s_l[w][r] * f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) acc[i] += sh.o[w][r][d0 + i] * f;
      }
      const int out_r = row0 + 8 * nt + r;
      if (!part.whole()) {   // the pair goes on in other CTAs: [dim][row]
        const int64_t slot = me == shares.owner(part.place(0)) ? 2 * me + 1 : 2 * me;
#pragma unroll
        for (int i = 0; i < kPer; ++i) a.part_o[(slot * HD + d0 + i) * G::kSlotRows + 8 * nt + r] = acc[i];
        if (d0 == 0) a.part_ml[slot * G::kSlotRows + 8 * nt + r] = make_float2(top, sum);
      } else if (out_r < rows) {
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
    }
  }
}

template <int HD, int NT>
cudaError_t launch(const TreeLaunch& a, int ctas, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, tree_e2m1_kernel<HD, NT>, a);
}

}  // namespace

cudaError_t launch_tree_e2m1(const TreeLaunch& a, const kvprm_cache& c, int tiles, int ctas, cudaStream_t stream) {
  const bool wide = c.head_dim == 128;
  if (tiles == 1) return wide ? launch<128, 1>(a, ctas, stream) : launch<64, 1>(a, ctas, stream);
  if (tiles == 2) return wide ? launch<128, 2>(a, ctas, stream) : launch<64, 2>(a, ctas, stream);
  return wide ? launch<128, 4>(a, ctas, stream) : launch<64, 4>(a, ctas, stream);
}

}  // namespace kvprm
