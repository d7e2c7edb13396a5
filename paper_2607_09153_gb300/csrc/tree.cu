// Attention of drafted tokens over the paged cache in tiles of 16 or 32 query rows (row = drafted token and head of the kv
// head's group): warp-level matrix instructions on fragments that are loaded straight from the pages.
//
// Each warp takes every fourth 16-token block of its CTA's part of a pair (tree.h) and keeps its own online softmax; the
// four meet at the part's end.  A lane's 16-byte loads are its operand fragments: the products q . k run over head
// dimensions in any order, so a lane takes consecutive ones for both operands, and the output's columns are named by the
// dimensions that its values' loads held.  Only the queries (the same for all warps) lie in shared memory; nothing waits
// at a barrier while the cache streams.
//
// 8-bit codes become fp16 in registers (one instruction for two; to bf16 it takes nine for four: 8 x 32,768 tokens of 8 kv
// heads 129 us, so 113), once for both tiles of 32 rows.  What fp16 lacks in range is kept beside it as powers of two: a query row is
// scaled to a largest magnitude of 1 to 2 (exact but for elements 2^-14 of that and smaller, which lose what is below
// 2^-25 of it), a key row's power multiplies the scores in fp32, and a value row's multiplies the weights, relative to the
// largest one met, E: a weight p becomes p 2^(e - E + 10), whose fp16 steps end at 2^-34 of a full weight's.  A page with a
// power below 2^-10 of E takes its values' product in bf16 instead, whose range is fp32's: its weights would lose what E,
// which may stand for a row that is not looked at, leaves out.
//
// What bounds it, measured on a GB300, a drafted token per sequence: a bf16 cache memory (8 kv heads of 128, 4 query heads
// each, 8 x 32,768 tokens in 168 us, 6,390 GB/s), an 8-bit one a page's instructions and its values' latency (the same in 107
// us, 5,040 GB/s; with 7 query heads each over 64 ragged sequences 75 us, 4,500 GB/s).  Loads two pages ahead did not help,
// in registers (100: they share scoreboards) or by asynchronous copies (79), nor did a fourth CTA.
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
// A running maximum may be exceeded by so many powers of two (of fp16 weights times 2^12 less, to stay below 65504).
constexpr float margin(bool e4m3) { return e4m3 ? 3.f : 8.f; }

__device__ __forceinline__ uint4 ldg_stream(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}
__device__ __forceinline__ uint4 ldg_stream2(const void* p) {   // 8 bytes
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// The low or the high two e4m3 codes of a word as fp16 (exact, in one instruction).
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
// mma_bf16_16816 (ptx.cuh) on fp16 operands.
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                              uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t bf16_of_f16(uint32_t v) {   // exact for codes
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
  return pack_bf16(f.x, f.y);
}
__device__ __forceinline__ float power_of(int field) { return __uint_as_float(static_cast<uint32_t>(field) << 23); }

// Whether one of two bf16 is infinite or NaN; whether one of four bytes is 255.
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}
__device__ __forceinline__ bool has_255(uint32_t w) { return ((~w - 0x01010101u) & w & 0x80808080u) != 0u; }
// A row's power of two from byte k of a word of exponents (255, NaN, is looked for before).
__device__ __forceinline__ float power(uint32_t w, int k) {
  const uint32_t bits = (k < 3 ? w << (23 - 8 * k) : w >> 1) & 0x7F800000u;
  return __uint_as_float(max(bits, 0x00400000u));
}

template <int HD, bool E4M3, int TILES>
__global__ void __launch_bounds__(kThreads, tree_rows_per_sm(TILES))
    tree_rows_kernel(const __grid_constant__ TreeLaunch a) {
  using G = TreeRows<TILES>;
  constexpr int KS = HD / 16;                       // 16-dim steps of q . k
  constexpr int NT = HD / 8;                        // 8-dim tiles of the output
  constexpr int kK = E4M3 ? HD / 64 : HD / 32;      // a lane's 16-byte pieces of a key row
  constexpr int kV = E4M3 ? 1 : HD / 64;            // of a value row (of 8 bytes with 64 codes)
  constexpr int kSize = E4M3 ? 1 : 2;
  __shared__ int32_t s_off[kTreeSeqs + 1];
  __shared__ int32_t s_sum[kWarps];
  __shared__ union {
    struct {
      uint4 bf16[TILES][KS][32];                              // the queries' fragments, by lane
      uint4 fp16[E4M3 ? TILES : 1][E4M3 ? KS : 1][32];        // and, for codes, scaled
    } q;
    float o[kWarps][16][HD + 1];                              // at a part's end, the warps' outputs
  } sh;
  auto& s_q = sh.q.bf16;
  auto& s_qh = sh.q.fp16;
  auto& s_o = sh.o;
  __shared__ float s_most[TILES][16][HD / 32];      // largest magnitude of 32 dims of a query row
  __shared__ float s_m[kWarps][16], s_l[kWarps][16];
  grid_dep_launch();
  tree_line<G, kThreads, HD>(a, s_off, s_sum);
  const int32_t total = s_off[a.n_seqs];
  if (total == 0) return;
  const TreeShares shares(total, gridDim.x, a.weight_full);
  const int me = blockIdx.x;
  tree_leave_line(a, s_off, shares.ctas);
  if (me >= shares.ctas) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, c = lane & 3;
  const int64_t head_bytes = static_cast<int64_t>(kTreePage) * HD * kSize, page_bytes = 2 * a.n_kv * head_bytes;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  int32_t u = shares.begin(me);
  const int32_t u_end = shares.begin(me + 1);
  int s_at = tree_find(s_off, a.n_seqs, u);
  TreePart part;
  while (tree_next<G>(a, s_off, u, u_end, s_at, part)) {
    const TreeSeq& q = part.q;
    const int g = part.g, row0 = part.tp * G::kSlotRows, rows = q.drafts * a.group;
    const int32_t* table = a.t.block_table + static_cast<int64_t>(a.seq0 + s_at) * a.t.max_blocks;
    const uint8_t* keys = a.pages + g * head_bytes;
    const uint8_t* values = keys + a.n_kv * head_bytes;
    const uint8_t* exponents = a.exponents + g * kTreePage;

    // ---- query fragments: rows gid and gid + 8 of a tile; warp w dims 32 w .. (two steps)
    __syncthreads();   // the last part's have been read
    float rs[TILES][2];   // what a row's scores are to be multiplied by
    {
      uint4 f[TILES][2];
#pragma unroll
      for (int ti = 0; ti < TILES; ++ti) {
        f[ti][0] = f[ti][1] = zero;
        if (warp >= HD / 32) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = row0 + 16 * ti + gid + 8 * h;
          uint4 v = zero;
          if (r < rows) {
            const int tok = tree_token(a, r);
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.t.q) + (q.start + static_cast<int64_t>(tok)) * a.t.q_token +
                                       (g * a.group + r - tok * a.group) * a.t.q_head;
            // bf16 keys: 8 dims from 32 w + 8 c on; codes: half of 16 dims from 64 (w / 2) + 16 c on
            v = __ldg(reinterpret_cast<const uint4*>(src + (E4M3 ? 64 * (warp >> 1) + 16 * c + 8 * (warp & 1) : 32 * warp + 8 * c)));
          }
          (h ? f[ti][0].y : f[ti][0].x) = v.x;
          (h ? f[ti][0].w : f[ti][0].z) = v.y;
          (h ? f[ti][1].y : f[ti][1].x) = v.z;
          (h ? f[ti][1].w : f[ti][1].z) = v.w;
          if (E4M3) {
            float most = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t x = word(v, k);
              most = fmaxf(most, fmaxf(fabsf(__uint_as_float(x << 16)), fabsf(__uint_as_float(x & 0xFFFF0000u))));
            }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            if (c == 0) s_most[ti][gid + 8 * h][warp] = most;
          }
        }
        s_q[ti][2 * warp][lane] = f[ti][0];
        s_q[ti][2 * warp + 1][lane] = f[ti][1];
      }
      __syncthreads();
      if constexpr (E4M3) {
#pragma unroll
        for (int ti = 0; ti < TILES; ++ti) {
          float up[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float most = 0.f;
#pragma unroll
            for (int k = 0; k < HD / 32; ++k) most = fmaxf(most, s_most[ti][gid + 8 * h][k]);
            int e = static_cast<int>(__float_as_uint(most) >> 23);   // (infinite or all zero: any scale does)
            e = e < 1 || e > 253 ? 127 : e;
            rs[ti][h] = power_of(e);
            up[h] = power_of(254 - e);
          }
          if (warp < HD / 32) {
            auto scaled = [&](uint32_t x, float by) {
              return pack_f16(__uint_as_float(x << 16) * by, __uint_as_float(x & 0xFFFF0000u) * by);
            };
#pragma unroll
            for (int k = 0; k < 2; ++k)
              s_qh[ti][2 * warp + k][lane] = make_uint4(scaled(f[ti][k].x, up[0]), scaled(f[ti][k].y, up[1]),
                                                        scaled(f[ti][k].z, up[0]), scaled(f[ti][k].w, up[1]));
          }
        }
        __syncthreads();
      } else {
#pragma unroll
        for (int ti = 0; ti < TILES; ++ti) rs[ti][0] = rs[ti][1] = 1.f;
      }
    }

    float o[TILES][NT][4], m[TILES][2], l[TILES][2];
#pragma unroll
    for (int ti = 0; ti < TILES; ++ti) {
#pragma unroll
      for (int i = 0; i < NT; ++i) o[ti][i][0] = o[ti][i][1] = o[ti][i][2] = o[ti][i][3] = 0.f;
      m[ti][0] = m[ti][1] = -INFINITY;
      l[ti][0] = l[ti][1] = 0.f;
    }
    bool poison = q.bad;        // of all rows of the sequence
    uint32_t poison_row = 0;    // bit 2 ti + h: of row gid + 8 h of tile ti
    // E, the exponent byte that the weights are relative to (from the first page on, at least 64: 2^-63; 0: none yet), and
    // 2^(10 + 127 - E), which the outputs are multiplied by
    int top_e = 0;
    float rel = 1.f;

    // One block's softmax step for one tile: scores s in units of log2 (token 2 c + (i & 1) + 8 n of row gid + 8 (i >> 1))
    // become the weights as an operand, the running maximum, sum and output following.  The maximum moves only when
    // a score passes it by more than a margin (the weights then stay below 2^margin, and most blocks need no exchange
    // between lanes).  The weights are rounded to bf16 or fp16, the values' type: their sum is not.
    auto softmax = [&](int ti, float(&s)[2][4], const float(&vf)[4], uint32_t(&pa)[4], bool fp16) {
      float mx[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) mx[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      if (__any_sync(0xffffffffu, mx[0] > m[ti][0] + margin(E4M3) || mx[1] > m[ti][1] + margin(E4M3))) {
        float al[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
          mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
          mx[h] = fmaxf(mx[h], m[ti][h]);
          al[h] = mx[h] == m[ti][h] ? 1.f : ex2_ftz(m[ti][h] - mx[h]);
          m[ti][h] = mx[h];
          l[ti][h] *= al[h];
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          o[ti][i][0] *= al[0];
          o[ti][i][1] *= al[0];
          o[ti][i][2] *= al[1];
          o[ti][i][3] *= al[1];
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float nm = m[ti][h] == -INFINITY ? 0.f : -m[ti][h];   // nothing seen yet: every score is -infinity
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float p0 = ex2_ftz(s[n][2 * h] + nm), p1 = ex2_ftz(s[n][2 * h + 1] + nm);
          l[ti][h] += p0 + p1;
          const float w0 = E4M3 ? p0 * vf[2 * n] : p0, w1 = E4M3 ? p1 * vf[2 * n + 1] : p1;
          pa[2 * n + h] = E4M3 && fp16 ? pack_f16(w0, w1) : pack_bf16(w0, w1);
        }
      }
    };

    const int c_end = min(part.c1, q.cached_blocks);
    uint4 kr[2][kK];
    auto page_of = [&](int b) { return b < c_end ? __ldg(table + b) : 0; };
    auto in_cache = [&](int32_t page) { return page >= 0 && page < a.n_pages; };
    auto load_keys = [&](int32_t page) {
      const uint8_t* base = keys + (in_cache(page) ? page : 0) * page_bytes + gid * HD * kSize + 16 * c;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < kK; ++j) kr[n][j] = a.n_pages > 0 ? ldg_stream(base + (8 * n * HD * kSize + 64 * j)) : zero;
    };

    uint32_t e4[4] = {0u, 0u, 0u, 0u};   // (as loaded: to put them together is to wait for them)
    auto load_exponents = [&](int32_t page) {
      if constexpr (E4M3) {
        if (a.n_pages == 0) return;
        const uint8_t* e = exponents + (in_cache(page) ? page : 0) * static_cast<int64_t>(2 * a.n_kv) * kTreePage + 2 * c;
        e4[0] = __ldg(reinterpret_cast<const uint16_t*>(e));
        e4[1] = __ldg(reinterpret_cast<const uint16_t*>(e + 8));
        e += a.n_kv * kTreePage;
        e4[2] = __ldg(reinterpret_cast<const uint16_t*>(e));
        e4[3] = __ldg(reinterpret_cast<const uint16_t*>(e + 8));
      }
    };

    // ---- the cache: pages b, b + 4, ..; the next page's keys and exponents and the page's own values are on their way while
    // scores are made
    int b = part.c0 + warp;
    int32_t page = page_of(b), next = page_of(b + kWarps);
    if (b < c_end) {
      load_keys(page);
      load_exponents(page);
    }
    for (; b < c_end; b += kWarps) {
      const int32_t after = page_of(b + 2 * kWarps);
      const int have = q.len - b * kTreePage;   // tokens of the page: 16 or more where it is full
      poison = poison || !in_cache(page);
      const int64_t at = (in_cache(page) ? page : 0) * static_cast<int64_t>(2 * a.n_kv);
      uint4 v[4][kV];
      uint32_t ke = e4[0] | e4[1] << 16, ve = e4[2] | e4[3] << 16;   // exponents of tokens 2 c, 2 c + 1, 8 + 2 c, 9 + 2 c
      {
        const uint8_t* base = values + at * head_bytes + (E4M3 ? gid * (HD / 8) : 16 * gid);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint8_t* p = base + (2 * c + (k & 1) + 8 * (k >> 1)) * HD * kSize;
#pragma unroll
          for (int h = 0; h < kV; ++h)
            v[k][h] = a.n_pages > 0 ? (E4M3 && HD == 64 ? ldg_stream2(p) : ldg_stream(p + 128 * h)) : zero;
        }
      }
      float s[TILES][2][4];
#pragma unroll
      for (int ti = 0; ti < TILES; ++ti)
#pragma unroll
        for (int n = 0; n < 2; ++n) s[ti][n][0] = s[ti][n][1] = s[ti][n][2] = s[ti][n][3] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t b0[2], b1[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          if constexpr (E4M3) {
            const uint32_t x = word(kr[n][k / 4], k % 4);
            b0[n] = codes_lo(x);
            b1[n] = codes_hi(x);
          } else {
            b0[n] = word(kr[n][k / 2], 2 * (k % 2));
            b1[n] = word(kr[n][k / 2], 2 * (k % 2) + 1);
          }
        }
#pragma unroll
        for (int ti = 0; ti < TILES; ++ti) {
          const uint4 f = E4M3 ? s_qh[E4M3 ? ti : 0][E4M3 ? k : 0][lane] : s_q[ti][k][lane];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            if constexpr (E4M3)
              mma_f16_16816(s[ti][n], f.x, f.y, f.z, f.w, b0[n], b1[n]);
            else
              mma_bf16_16816(s[ti][n], f.x, f.y, f.z, f.w, b0[n], b1[n]);
          }
        }
      }
      if (b + kWarps < c_end) {
        load_keys(next);
        load_exponents(next);
      }
      if (have < kTreePage) {   // the last page: its places beyond the length may hold anything, even NaN
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int tok = 2 * c + (k & 1) + 8 * (k >> 1);
          if (tok < have) continue;
#pragma unroll
          for (int h = 0; h < kV; ++h) v[k][h] = zero;
          ke = (ke & ~(255u << (8 * k))) | 1u << (8 * k);
          ve = (ve & ~(255u << (8 * k))) | 1u << (8 * k);
        }
      }
      bool wide = false;   // a value row's power far below E
      if constexpr (E4M3) {
        // a value row's power beyond E + 2 (NaN among them): E moves there and the outputs with it
        const uint32_t most = max(max(ve & 255u, (ve >> 8) & 255u), max((ve >> 16) & 255u, ve >> 24));
        const uint32_t least = min(min(ve & 255u, (ve >> 8) & 255u), min((ve >> 16) & 255u, ve >> 24));
        if (__any_sync(0xffffffffu, static_cast<int>(most) > top_e + 2 || static_cast<int>(least) < top_e - 10 || has_255(ke)) ||
            top_e == 0) {
          if (__any_sync(0xffffffffu, has_255(ke) || has_255(ve))) poison = true;   // every row sees the page
          uint32_t e = most;
          e = max(e, __shfl_xor_sync(0xffffffffu, e, 1));
          e = max(e, __shfl_xor_sync(0xffffffffu, e, 2));
          const int now = max(min(static_cast<int>(e), 254), max(top_e, 64));
          const float f = power_of(max(127 + top_e - now, 0));
#pragma unroll
          for (int ti = 0; ti < TILES; ++ti)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
              for (int k = 0; k < 4; ++k) o[ti][i][k] *= f;
          top_e = now;
          rel = power_of(264 - now);
          wide = __any_sync(0xffffffffu, static_cast<int>(least) < now - 10);
        }
      }
      float kf[4], vf[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        kf[k] = E4M3 ? power(ke, k) * a.scale_log2 : a.scale_log2;
        vf[k] = E4M3 ? power(ve, k) * rel : 1.f;
      }
      uint32_t pa[TILES][4];
#pragma unroll
      for (int ti = 0; ti < TILES; ++ti) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = s[ti][n][i] * (E4M3 ? kf[2 * n + (i & 1)] * rs[ti][i >> 1] : kf[0]);
            s[ti][n][i] = have < kTreePage && 2 * c + (i & 1) + 8 * n >= have ? -INFINITY : x;   // (a scale may be negative)
          }
        softmax(ti, s[ti], vf, pa[ti], !wide);
      }
      // the weights' product with the values
      auto product = [&](auto codes) {
#pragma unroll
        for (int w = 0; w < NT / 4; ++w) {   // four 8-dim tiles: a word of codes, or two words of bf16, of each of the lane's tokens
          uint32_t b0[4], b1[4];
          if constexpr (E4M3) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t t0 = __byte_perm(word(v[0][0], w), word(v[1][0], w), x ? 0x7362 : 0x5140);   // tokens side by side
              const uint32_t t1 = __byte_perm(word(v[2][0], w), word(v[3][0], w), x ? 0x7362 : 0x5140);
              b0[2 * x] = codes_lo(t0);
              b0[2 * x + 1] = codes_hi(t0);
              b1[2 * x] = codes_lo(t1);
              b1[2 * x + 1] = codes_hi(t1);
            }
          } else {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int at_word = 2 * (w & 1) + (x >> 1), sel = x & 1 ? 0x7632 : 0x5410;
              b0[x] = __byte_perm(word(v[0][w / 2], at_word), word(v[1][w / 2], at_word), sel);
              b1[x] = __byte_perm(word(v[2][w / 2], at_word), word(v[3][w / 2], at_word), sel);
            }
          }
#pragma unroll
          for (int ti = 0; ti < TILES; ++ti)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              float(&d)[4] = o[ti][4 * w + x];
              if constexpr (decltype(codes)::value)
                mma_f16_16816(d, pa[ti][0], pa[ti][1], pa[ti][2], pa[ti][3], b0[x], b1[x]);
              else if constexpr (E4M3)
                mma_bf16_16816(d, pa[ti][0], pa[ti][1], pa[ti][2], pa[ti][3], bf16_of_f16(b0[x]), bf16_of_f16(b1[x]));
              else
                mma_bf16_16816(d, pa[ti][0], pa[ti][1], pa[ti][2], pa[ti][3], b0[x], b1[x]);
            }
        }
      };
      if (E4M3 && !wide)
        product(std::integral_constant<bool, E4M3>());
      else
        product(std::false_type());
      page = next;
      next = after;
    }

    // ---- drafted tokens: bf16 rows of their own tensors, whatever the cache holds (b is the warp's next block after the cache)
    if (E4M3 && top_e == 0) {
      top_e = 127;
      rel = power_of(137);
    }
    for (; b < part.c1; b += kWarps) {
      const int j0 = (b - q.cached_blocks) * kTreePage, have = q.drafts - j0;
      const __nv_bfloat16* kd = static_cast<const __nv_bfloat16*>(a.t.k) + (q.start + static_cast<int64_t>(j0)) * a.t.k_token + g * a.t.k_head;
      const __nv_bfloat16* vd = static_cast<const __nv_bfloat16*>(a.t.v) + (q.start + static_cast<int64_t>(j0)) * a.t.v_token + g * a.t.v_head;
      float s[TILES][2][4];
#pragma unroll
      for (int ti = 0; ti < TILES; ++ti)
#pragma unroll
        for (int n = 0; n < 2; ++n) s[ti][n][0] = s[ti][n][1] = s[ti][n][2] = s[ti][n][3] = 0.f;
#pragma unroll 1
      for (int j = 0; j < HD / 32; ++j) {   // two steps
        uint4 x[2];
#pragma unroll
        for (int n = 0; n < 2; ++n)
          x[n] = 8 * n + gid < have ? __ldg(reinterpret_cast<const uint4*>(
                                          kd + (8 * n + gid) * a.t.k_token +
                                          (E4M3 ? 64 * (j >> 1) + 16 * c + 8 * (j & 1) : 32 * j + 8 * c)))
                                    : zero;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int ti = 0; ti < TILES; ++ti) {
            const uint4 f = s_q[ti][2 * j + k][lane];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const uint32_t lo = word(x[n], 2 * k), hi = word(x[n], 2 * k + 1);
              mma_bf16_16816(s[ti][n], f.x, f.y, f.z, f.w, lo, hi);
            }
          }
      }
      constexpr int kD = HD / 64;   // 16-byte pieces of a lane's dims of one value row
      uint4 v[4][kD];
      uint32_t bad = 0;   // tokens whose value row is not finite
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int tok = 2 * c + (k & 1) + 8 * (k >> 1);
        bool off = false;
#pragma unroll
        for (int d = 0; d < kD; ++d) {
          const int dim = E4M3 ? gid * (HD / 8) + 8 * d : 64 * d + 8 * gid;
          v[k][d] = tok < have ? __ldg(reinterpret_cast<const uint4*>(vd + tok * a.t.v_token + dim)) : zero;
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
      uint32_t pa[TILES][4];
#pragma unroll
      for (int ti = 0; ti < TILES; ++ti) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = row0 + 16 * ti + gid + 8 * h;
          const uint32_t sees = r < rows ? tree_sees16(a, q, tree_token(a, r), j0) : 0u;
          if (sees & bad) poison_row |= 1u << (2 * ti + h);
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              s[ti][n][2 * h + i] = (sees >> (2 * c + i + 8 * n)) & 1u ? s[ti][n][2 * h + i] * a.scale_log2 : -INFINITY;
        }
        const float same[4] = {rel, rel, rel, rel};
        softmax(ti, s[ti], same, pa[ti], false);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int d = i / 8, w = (i % 8) >> 1;
        const uint32_t sel = i & 1 ? 0x7632 : 0x5410;
        const uint32_t b0 = __byte_perm(word(v[0][d], w), word(v[1][d], w), sel);
        const uint32_t b1 = __byte_perm(word(v[2][d], w), word(v[3][d], w), sel);
#pragma unroll
        for (int ti = 0; ti < TILES; ++ti) mma_bf16_16816(o[ti][i], pa[ti][0], pa[ti][1], pa[ti][2], pa[ti][3], b0, b1);
      }
    }

    // ---- the part's end: the four warps' states meet, 16 rows at a time
    const float down = power_of(max(top_e - 10, 1));   // 1 / rel
#pragma unroll
    for (int ti = 0; ti < TILES; ++ti) {
      __syncthreads();   // the queries (or the last 16 rows) have been read
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = l[ti][h];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (poison || (poison_row >> (2 * ti + h)) & 1u) sum = NAN;
        if (c == 0) {
          s_m[warp][gid + 8 * h] = m[ti][h];
          s_l[warp][gid + 8 * h] = sum;
        }
      }
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {   // column 2 c + (e & 1) of tile i: the dimension that its values' load held
          const int n = 2 * c + (e & 1);
          const int dim = E4M3 ? n * (HD / 8) + i : 64 * (i / 8) + 8 * n + i % 8;
          s_o[warp][gid + 8 * (e >> 1)][dim] = E4M3 ? o[ti][i][e] * down : o[ti][i][e];
        }
      __syncthreads();
      constexpr int kPer = 16 * HD / kThreads;   // outputs of a thread: part of one row
      const int r = threadIdx.x % 16, d0 = threadIdx.x / 16 * kPer;
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
      const int out_r = row0 + 16 * ti + r;
      if (!part.whole()) {   // the pair goes on in other CTAs: [dim][row]
        const int64_t slot = me == shares.owner(part.place(0)) ? 2 * me + 1 : 2 * me;
#pragma unroll
        for (int i = 0; i < kPer; ++i) a.part_o[(slot * HD + d0 + i) * G::kSlotRows + 16 * ti + r] = acc[i];
        if (d0 == 0) a.part_ml[slot * G::kSlotRows + 16 * ti + r] = make_float2(top, sum);
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
}

template <int HD, bool E4M3, int TILES>
cudaError_t launch(const TreeLaunch& a, int ctas, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, tree_rows_kernel<HD, E4M3, TILES>, a);
}

}  // namespace

cudaError_t launch_tree_rows(const TreeLaunch& a, const kvprm_cache& c, int tiles, int ctas, cudaStream_t stream) {
  const bool wide = c.head_dim == 128, codes = c.format == KVPRM_CACHE_E4M3;
  if (tiles == 2)
    return codes ? (wide ? launch<128, true, 2>(a, ctas, stream) : launch<64, true, 2>(a, ctas, stream))
                 : (wide ? launch<128, false, 2>(a, ctas, stream) : launch<64, false, 2>(a, ctas, stream));
  return codes ? (wide ? launch<128, true, 1>(a, ctas, stream) : launch<64, true, 1>(a, ctas, stream))
               : (wide ? launch<128, false, 1>(a, ctas, stream) : launch<64, false, 1>(a, ctas, stream));
}

}  // namespace kvprm
