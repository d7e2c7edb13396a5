// Attention of drafted tokens over the paged cache, in tiles of 16 query rows (row = drafted token and
// head of the kv head's group): warp-level matrix instructions on fragments that are loaded straight
// from the pages.
//
// Each warp takes every fourth 16-token block of its CTA's part of a pair (tree.h) and keeps its own
// online softmax; the four meet at the part's end.  A lane's 16-byte loads are its operand fragments:
// the products q . k run over head dimensions in any order, so a lane takes consecutive ones for both
// operands, and the output's columns are named by the dimensions that its values' loads held.  Nothing
// goes through shared memory or waits at a barrier while the cache streams.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ptx.cuh"
#include "rope.h"
#include "tree.h"

namespace kvprm {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kRows = 16;
constexpr float kMargin = 8.f;   // a running maximum may be exceeded by so many powers of two

__device__ __forceinline__ uint4 ldg_stream(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}
__device__ __forceinline__ uint2 ldg_stream2(const void* p) {
  uint2 r;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Two e4m3 codes as bf16: the even or the odd bytes of a word.  A code's exponent and mantissa at bf16's
// place are 2^-120 of its value (the biases differ by 120), subnormals included.
__device__ __forceinline__ uint32_t rebias(uint32_t v) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0x7B807B80u));   // 2^120
  return r;
}
__device__ __forceinline__ uint32_t e4m3_even(uint32_t w) {
  return rebias(((w << 4) & 0x07F007F0u) | ((w << 8) & 0x80008000u));
}
__device__ __forceinline__ uint32_t e4m3_odd(uint32_t w) { return rebias(((w >> 4) & 0x07F007F0u) | (w & 0x80008000u)); }

// Whether one of two bf16 is infinite or NaN.
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

template <int HD, bool E4M3>
struct Frag {
  // keys: one or two 16-byte loads per token and 64 dims; values: 16 bytes per 64 dims (bf16), HD / 8 bytes (e4m3)
  static constexpr int kK = E4M3 ? HD / 64 : HD / 32;
  static constexpr int kV = E4M3 ? 1 : HD / 64;
};

template <int HD, bool E4M3>
__global__ void __launch_bounds__(kThreads, kTreeRows16PerSm) tree_rows16_kernel(const __grid_constant__ TreeLaunch a) {
  using F = Frag<HD, E4M3>;
  constexpr int KS = HD / 16;   // 16-dim steps of q . k
  constexpr int NT = HD / 8;    // 8-dim tiles of the output
  __shared__ int32_t s_off[kTreeSeqs + 1];
  __shared__ int32_t s_sum[kWarps];
  __shared__ float s_o[kWarps][kRows][HD + 1];
  __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
  grid_dep_launch();
  tree_line<TreeRows16, kThreads>(a, s_off, s_sum);
  const int32_t total = s_off[a.n_seqs];
  if (total == 0) return;
  const TreeShares shares(total, gridDim.x, a.weight_full);
  const int me = blockIdx.x;
  tree_leave_line(a, s_off, shares.ctas);
  if (me >= shares.ctas) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, c = lane & 3;
  const int64_t block_bytes = static_cast<int64_t>(kTreePage) * HD * (E4M3 ? 1 : 2);   // of one head's keys
  int32_t u = shares.begin(me);
  const int32_t u_end = shares.begin(me + 1);
  int s = tree_find(s_off, a.n_seqs, u);
  TreePart part;
  for (bool first_part = true; tree_next<TreeRows16>(a, s_off, u, u_end, s, part); first_part = false) {
    if (!first_part) __syncthreads();   // the last part's states have been read
    const TreeSeq& q = part.q;
    const int g = part.g, tile = part.tp, rows = q.drafts * a.group;
    const int32_t* table = a.t.block_table + static_cast<int64_t>(a.seq0 + s) * a.t.max_blocks;

    // ---- query fragments: rows gid and gid + 8
    uint32_t qa[KS][4];
    int row_t[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = tile * kRows + gid + 8 * h;
      const bool live = r < rows;
      row_t[h] = live ? tree_token(a, r) : -1;
      const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.t.q) +
                                 (live ? (q.start + static_cast<int64_t>(row_t[h])) * a.t.q_token +
                                             (g * a.group + r - row_t[h] * a.group) * a.t.q_head
                                       : 0);
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
      if constexpr (E4M3) {
#pragma unroll
        for (int j = 0; j < HD / 64; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 v = live ? __ldg(reinterpret_cast<const uint4*>(src + 64 * j + 16 * c + 8 * i)) : zero;
#pragma unroll
            for (int k = 0; k < 2; ++k) {   // dims of a word: even ones, odd ones
              const uint32_t lo = word(v, 2 * k), hi = word(v, 2 * k + 1);
              qa[4 * j + 2 * i + k][h] = __byte_perm(lo, hi, 0x5410);
              qa[4 * j + 2 * i + k][2 + h] = __byte_perm(lo, hi, 0x7632);
            }
          }
      } else {
#pragma unroll
        for (int j = 0; j < HD / 32; ++j) {
          const uint4 v = live ? __ldg(reinterpret_cast<const uint4*>(src + 32 * j + 8 * c)) : zero;
          qa[2 * j][h] = v.x;
          qa[2 * j][2 + h] = v.y;
          qa[2 * j + 1][h] = v.z;
          qa[2 * j + 1][2 + h] = v.w;
        }
      }
    }

    float o[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    bool poison = q.bad;        // of all rows of the sequence
    bool poison_row[2] = {false, false};

    // ---- one block's fragments
    struct KeyRegs {
      uint4 k[2][F::kK];
    } kr;
    auto page_of = [&](int b) -> int64_t {   // -1: not a page of the cache
      const int32_t p = __ldg(table + b);
      return p >= 0 && p < a.n_pages ? p : -1;
    };
    auto draft_row = [&](const void* base, int64_t tok, int64_t head, int j) {
      return static_cast<const __nv_bfloat16*>(base) + (q.start + static_cast<int64_t>(j)) * tok + g * head;
    };
    auto load_keys = [&](int64_t page) {
      const uint8_t* base = a.pages + (page * 2 * a.n_kv + g) * block_bytes;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < F::kK; ++j) {
          const int at = (8 * n + gid) * HD * (E4M3 ? 1 : 2) + 64 * j + 16 * c;
          kr.k[n][j] = page >= 0 ? ldg_stream(base + at) : make_uint4(0u, 0u, 0u, 0u);
        }
    };

    // One block's softmax step: raw scores s (token 2 c + (i & 1) + 8 n of row gid + 8 (i >> 1)) and the tokens that the
    // rows see become the weights as an operand, the running maximum, sum and output following.  The maximum moves
    // only when a score passes it by more than kMargin (the weights then stay below 2^kMargin, and most blocks need
    // no exchange between lanes).  The weights are rounded to bf16, the values' type: their sum is not.
    auto softmax = [&](float(&s)[2][4], const uint32_t(&sees)[2], const float(&vf)[4], uint32_t(&pa)[4]) {
      float mx[2];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[n][i] = (sees[i >> 1] >> (2 * c + (i & 1) + 8 * n)) & 1u ? s[n][i] * a.scale_log2 : -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h) mx[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      if (__any_sync(0xffffffffu, mx[0] > m[0] + kMargin || mx[1] > m[1] + kMargin)) {
        float al[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
          mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
          mx[h] = fmaxf(mx[h], m[h]);
          al[h] = mx[h] == m[h] ? 1.f : ex2_ftz(m[h] - mx[h]);
          m[h] = mx[h];
          l[h] *= al[h];
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          o[i][0] *= al[0];
          o[i][1] *= al[0];
          o[i][2] *= al[1];
          o[i][3] *= al[1];
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float nm = m[h] == -INFINITY ? 0.f : -m[h];   // nothing seen yet: every score is -infinity
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float p0 = ex2_ftz(s[n][2 * h] + nm), p1 = ex2_ftz(s[n][2 * h + 1] + nm);
          l[h] += p0 + p1;
          pa[2 * n + h] = pack_bf16(p0 * vf[2 * n], p1 * vf[2 * n + 1]);
        }
      }
    };

    const int b_end = part.c1;
    int b = part.c0 + warp;
    int64_t page = -1;
    if (b < min(b_end, q.cached_blocks)) {
      page = page_of(b);
      load_keys(page);
    }
    for (; b < b_end; b += kWarps) {
      const bool cached = b < q.cached_blocks;
      const int next = b + kWarps;
      const bool next_cached = next < min(b_end, q.cached_blocks);
      const int64_t next_page = next_cached ? page_of(next) : -1;
      const int j0 = cached ? b * kTreePage : (b - q.cached_blocks) * kTreePage;
      const int have = cached ? q.len - j0 : q.drafts - j0;   // tokens of the block, 16 or more where it is full
      float s[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
      uint32_t sees[2];   // tokens that rows gid and gid + 8 see
      if (cached) {
        poison = poison || page < 0;
        // values and the rows' powers of two on their way while the scores are made
        uint4 v[4][F::kV];
        uint4 ke, ve;
        {
          const uint8_t* base = a.pages + ((page * 2 + 1) * a.n_kv + g) * block_bytes;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int tok = 2 * c + (k & 1) + 8 * (k >> 1);
            const bool live = page >= 0 && tok < have;   // beyond the length: anything, even NaN
            if constexpr (E4M3) {
              const uint8_t* p = base + tok * HD + gid * (HD / 8);
              if constexpr (HD == 128) {
                v[k][0] = live ? ldg_stream(p) : make_uint4(0u, 0u, 0u, 0u);
              } else {
                const uint2 w = live ? ldg_stream2(p) : make_uint2(0u, 0u);
                v[k][0] = make_uint4(w.x, w.y, 0u, 0u);
              }
            } else {
#pragma unroll
              for (int h = 0; h < F::kV; ++h)
                v[k][h] = live ? ldg_stream(base + (tok * HD + 64 * h + 8 * gid) * 2) : make_uint4(0u, 0u, 0u, 0u);
            }
          }
          if constexpr (E4M3) {
            const uint8_t* e = a.exponents + (page * 2 * a.n_kv + g) * kTreePage;
            ke = page >= 0 ? __ldg(reinterpret_cast<const uint4*>(e)) : make_uint4(0u, 0u, 0u, 0u);
            ve = page >= 0 ? __ldg(reinterpret_cast<const uint4*>(e + static_cast<int64_t>(a.n_kv) * kTreePage))
                           : make_uint4(0u, 0u, 0u, 0u);
          }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int j = 0; j < F::kK; ++j) {
            if constexpr (E4M3) {
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const uint32_t x = word(kr.k[n][j], w);
                const uint32_t(&A)[4] = qa[4 * j + w];
                mma_bf16_16816(s[n], A[0], A[1], A[2], A[3], e4m3_even(x), e4m3_odd(x));
              }
            } else {
              const uint32_t(&A)[4] = qa[2 * j];
              const uint32_t(&B)[4] = qa[2 * j + 1];
              mma_bf16_16816(s[n], A[0], A[1], A[2], A[3], kr.k[n][j].x, kr.k[n][j].y);
              mma_bf16_16816(s[n], B[0], B[1], B[2], B[3], kr.k[n][j].z, kr.k[n][j].w);
            }
          }
        if (next_cached) load_keys(next_page);
        sees[0] = sees[1] = have >= 16 ? 0xFFFFu : (1u << have) - 1u;
        float vf[4] = {1.f, 1.f, 1.f, 1.f};
        if constexpr (E4M3) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int tok = 2 * c + (k & 1) + 8 * (k >> 1);
            const uint32_t kw = word(ke, (tok >> 2)), vw = word(ve, (tok >> 2));
            const float kf = row_factor((kw >> (8 * (tok & 3))) & 0xFFu);
            vf[k] = tok < have ? row_factor((vw >> (8 * (tok & 3))) & 0xFFu) : 0.f;
            s[k >> 1][k & 1] *= kf;
            s[k >> 1][2 + (k & 1)] *= kf;
          }
        }
        uint32_t pa[4];
        softmax(s, sees, vf, pa);
        if constexpr (E4M3) {
#pragma unroll
          for (int w = 0; w < HD / 32; ++w) {
            const uint32_t x0 = word(v[0][0], w), x1 = word(v[1][0], w), y0 = word(v[2][0], w), y1 = word(v[3][0], w);
            const uint32_t a0 = __byte_perm(x0, x1, 0x5410), a1 = __byte_perm(x0, x1, 0x7632);
            const uint32_t c0 = __byte_perm(y0, y1, 0x5410), c1 = __byte_perm(y0, y1, 0x7632);
            mma_bf16_16816(o[4 * w], pa[0], pa[1], pa[2], pa[3], e4m3_even(a0), e4m3_even(c0));
            mma_bf16_16816(o[4 * w + 1], pa[0], pa[1], pa[2], pa[3], e4m3_odd(a0), e4m3_odd(c0));
            mma_bf16_16816(o[4 * w + 2], pa[0], pa[1], pa[2], pa[3], e4m3_even(a1), e4m3_even(c1));
            mma_bf16_16816(o[4 * w + 3], pa[0], pa[1], pa[2], pa[3], e4m3_odd(a1), e4m3_odd(c1));
          }
        } else {
#pragma unroll
          for (int h = 0; h < F::kV; ++h)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t sel = i & 1 ? 0x7632 : 0x5410;
              mma_bf16_16816(o[8 * h + i], pa[0], pa[1], pa[2], pa[3],
                             __byte_perm(word(v[0][h], i >> 1), word(v[1][h], i >> 1), sel),
                             __byte_perm(word(v[2][h], i >> 1), word(v[3][h], i >> 1), sel));
            }
        }
      } else {
        // ---- drafted tokens: bf16 rows of their own tensors, whatever the cache holds
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int j = 8 * n + gid;
          const __nv_bfloat16* row = draft_row(a.t.k, a.t.k_token, a.t.k_head, j0 + j);
          if constexpr (E4M3) {
#pragma unroll
            for (int d = 0; d < HD / 64; ++d)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const uint4 x = j < have ? __ldg(reinterpret_cast<const uint4*>(row + 64 * d + 16 * c + 8 * i)) : zero;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const uint32_t(&A)[4] = qa[4 * d + 2 * i + k];
                  mma_bf16_16816(s[n], A[0], A[1], A[2], A[3], __byte_perm(word(x, 2 * k), word(x, 2 * k + 1), 0x5410),
                                 __byte_perm(word(x, 2 * k), word(x, 2 * k + 1), 0x7632));
                }
              }
          } else {
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
              const uint4 x = j < have ? __ldg(reinterpret_cast<const uint4*>(row + 32 * d + 8 * c)) : zero;
              const uint32_t(&A)[4] = qa[2 * d];
              const uint32_t(&B)[4] = qa[2 * d + 1];
              mma_bf16_16816(s[n], A[0], A[1], A[2], A[3], x.x, x.y);
              mma_bf16_16816(s[n], B[0], B[1], B[2], B[3], x.z, x.w);
            }
          }
        }
        constexpr int kD = HD / 64;   // 16-byte pieces of a lane's dims of one value row
        uint4 v[4][kD];
        uint32_t bad = 0;   // tokens whose value row is not finite
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int tok = 2 * c + (k & 1) + 8 * (k >> 1);
          const __nv_bfloat16* row = draft_row(a.t.v, a.t.v_token, a.t.v_head, j0 + tok);
          bool off = false;
#pragma unroll
          for (int d = 0; d < kD; ++d) {
            const int dim = E4M3 ? gid * (HD / 8) + 8 * d : 64 * d + 8 * gid;
            v[k][d] = tok < have ? __ldg(reinterpret_cast<const uint4*>(row + dim)) : zero;
            off = off || not_finite2(v[k][d].x) || not_finite2(v[k][d].y) || not_finite2(v[k][d].z) || not_finite2(v[k][d].w);
          }
          const uint32_t who = __ballot_sync(0xffffffffu, off);
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (who & (0x11111111u << x)) bad |= 1u << (2 * x + (k & 1) + 8 * (k >> 1));
          if ((bad >> tok) & 1u) {   // a weight of zero must leave no trace of it: rows that see it are marked instead
#pragma unroll
            for (int d = 0; d < kD; ++d) v[k][d] = zero;
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          sees[h] = row_t[h] >= 0 ? tree_sees16(a, q, row_t[h], j0) : 0u;
          poison_row[h] = poison_row[h] || (sees[h] & bad) != 0;
        }
        const float vf[4] = {1.f, 1.f, 1.f, 1.f};
        uint32_t pa[4];
        softmax(s, sees, vf, pa);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const int d = i / 8, w = (i % 8) >> 1;
          const uint32_t sel = i & 1 ? 0x7632 : 0x5410;
          mma_bf16_16816(o[i], pa[0], pa[1], pa[2], pa[3], __byte_perm(word(v[0][d], w), word(v[1][d], w), sel),
                         __byte_perm(word(v[2][d], w), word(v[3][d], w), sel));
        }
      }
      page = next_page;
    }

    // ---- the part's end: the four warps' states meet
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      if (poison || poison_row[h]) l[h] = NAN;
      if (c == 0) {
        s_m[warp][gid + 8 * h] = m[h];
        s_l[warp][gid + 8 * h] = l[h];
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {   // column 2 c + (e & 1) of tile i: the dimension that its values' load held
        const int n = 2 * c + (e & 1);
        const int dim = E4M3 ? n * (HD / 8) + i : 64 * (i / 8) + 8 * n + i % 8;
        s_o[warp][gid + 8 * (e >> 1)][dim] = o[i][e];
      }
    __syncthreads();
    constexpr int kPer = kRows * HD / kThreads;   // outputs of a thread: part of one row
    const int r = threadIdx.x % kRows, d0 = threadIdx.x / kRows * kPer;
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
      for (int i = 0; i < kPer; ++i) acc[i] += s_o[w][r][d0 + i] * f;
    }
    const int out_r = tile * kRows + r;
    if (!part.whole()) {   // the pair goes on in other CTAs
      const int slot = me == shares.owner(part.place(0)) ? 2 * me + 1 : 2 * me;
#pragma unroll
      for (int i = 0; i < kPer; ++i) a.part_o[(static_cast<int64_t>(slot) * HD + d0 + i) * kRows + r] = acc[i];
      if (d0 == 0) a.part_ml[slot * kRows + r] = make_float2(top, sum);
    } else if (out_r < rows) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that saw nothing: zeros; NaN stays
      const int tok = tree_token(a, out_r);
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.t.out) + (q.start + static_cast<int64_t>(tok)) * a.t.out_token +
                           (g * a.group + out_r - tok * a.group) * a.t.out_head + d0;
#pragma unroll
      for (int i = 0; i < kPer; i += 8) {
        uint4 w;
        w.x = pack_bf16(acc[i] * inv, acc[i + 1] * inv);
        w.y = pack_bf16(acc[i + 2] * inv, acc[i + 3] * inv);
        w.z = pack_bf16(acc[i + 4] * inv, acc[i + 5] * inv);
        w.w = pack_bf16(acc[i + 6] * inv, acc[i + 7] * inv);
        *reinterpret_cast<uint4*>(dst + i) = w;
      }
    }
  }
}

template <int HD, bool E4M3>
cudaError_t launch(const TreeLaunch& a, int ctas, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, tree_rows16_kernel<HD, E4M3>, a);
}

}  // namespace

cudaError_t launch_tree_rows16(const TreeLaunch& a, const kvprm_cache& c, int ctas, cudaStream_t stream) {
  if (c.head_dim == 128)
    return c.format == KVPRM_CACHE_E4M3 ? launch<128, true>(a, ctas, stream) : launch<128, false>(a, ctas, stream);
  return c.format == KVPRM_CACHE_E4M3 ? launch<64, true>(a, ctas, stream) : launch<64, false>(a, ctas, stream);
}

}  // namespace kvprm
