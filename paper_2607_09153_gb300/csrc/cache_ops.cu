// Rotary positions, and the paged cache written (bf16, or 8-bit floating point with a power of two
// per row) and expanded (8 bits to bf16): kvprm_rope_*, kvprm_cache_write, kvprm_cache_expand.
//
// All three move each element once and compute little, so they are bound by memory (large calls) or
// by one launch's latency (a decoding step).  What they share: a CTA takes a few tokens, makes each
// token's cosines and sines once in shared memory, and its threads then run over the tokens' heads.
// Measured on a GB300 (copy rate 6,773 GB/s): 32,768 tokens of 32 + 8 heads of 128 rotated in bf16 in
// 103 us (6,540 GB/s; with eight tokens a CTA 106; neighbouring pairs 110), 9,001 tokens of 16 + 4 heads
// of 64, fp32 gradients, in 20 us (4,500 GB/s: not two waves of CTAs, whose loads wait behind a barrier
// for their sines), 4,099 e4m3 pages of 8 heads expanded in 67 us (6,040 GB/s), 30,001 tokens of 8 heads
// rotated and written as e4m3 in 47 us (3,930 GB/s: a chain of slot, row, shuffles and store for each
// token of a thread, whose loads stall it most, with 0.62 of the issue slots in use; not rotated 39 us,
// from fp32 55, into bf16 pages 49).  Steps of 16 to 64 tokens take 2 to 2.5 us of the GPU's time.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "ptx.cuh"
#include "rope.h"

namespace kvprm {

namespace {
thread_local char g_message[256];
}  // namespace

int operator_fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_message, sizeof g_message, fmt, ap);
  va_end(ap);
  return code;
}

namespace {

constexpr int kThreads = 256;
constexpr int kRopeTokens = 4, kWriteTokens = 8;   // tokens of a CTA at most
constexpr int kMaxHeads = 1024, kMaxHeadDim = 512;

// ---------------------------------------------------------------- elements
template <typename T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f(float v) { return v; }
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

// N consecutive elements, 16 bytes at a time where VEC promises the alignment.
template <typename T, int N, bool VEC>
__device__ __forceinline__ void load_n(const T* p, float (&x)[N]) {
  if constexpr (VEC) {
    constexpr int kPer = 16 / sizeof(T);
    static_assert(N % kPer == 0, "whole 16-byte accesses");
#pragma unroll
    for (int i = 0; i < N / kPer; ++i) {
      const uint4 r = reinterpret_cast<const uint4*>(p)[i];   // not the read-only path: a rotation may be in place
      const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[i * kPer + k] = to_f<T>(e[k]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f<T>(p[i]);
  }
}
template <typename T, int N, bool VEC>
__device__ __forceinline__ void store_n(T* p, const float (&x)[N]) {
  if constexpr (VEC) {
    constexpr int kPer = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < N / kPer; ++i) {
      uint4 r;
      T* e = reinterpret_cast<T*>(&r);
#pragma unroll
      for (int k = 0; k < kPer; ++k) e[k] = from_f<T>(x[i * kPer + k]);
      reinterpret_cast<uint4*>(p)[i] = r;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = from_f<T>(x[i]);
  }
}

// Division by a number that a launch keeps: exact for n * d < 2^32 (8 tokens * kMaxHeads * kMaxHeadDim^2
// is the most that happens here).
struct FastDiv {
  uint32_t d, m;
  __host__ explicit FastDiv(uint32_t d_ = 1) : d(d_), m(d_ > 1 ? 0xFFFFFFFFu / d_ + 1u : 0u) {}
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return m ? __umulhi(n, m) : n; }
};

// Cosines and sines (times the magnitude) of a CTA's tokens, [token][pair] in shared memory.  The
// angle is pos * turns in whole numbers modulo one turn, which rounds nothing: it is off by the
// table's own error (2^-53 turns for each position at most), the lower half that is left out (2^-32)
// and a float's 24 bits (2^-26), where a 32-bit product of a position of 131,072 and a frequency would
// be 2^-8 radians off.
__device__ __forceinline__ void fill_rotations(const RopeTable& tab, const FastDiv& by_pairs, const int32_t* __restrict__ positions,
                                               int64_t first, int tokens, float sign, float* s_cos, float* s_sin) {
  const int pairs = tab.dim >> 1;
  for (int i = threadIdx.x; i < tokens * pairs; i += blockDim.x) {
    const int t = static_cast<int>(by_pairs.div(i)), pair = i - t * pairs;
    const uint64_t a = static_cast<uint64_t>(static_cast<int64_t>(__ldg(positions + first + t))) * tab.turns[pair];
    const float half_turns = static_cast<float>(static_cast<int32_t>(a >> 32)) * 0x1p-31f;
    float sn, cs;
    sincospif(half_turns, &sn, &cs);
    s_cos[i] = cs * tab.magnitude;
    s_sin[i] = sn * (sign * tab.magnitude);
  }
}

// ---------------------------------------------------------------- rotation
struct RopeLaunch {
  RopeTable tab;
  kvprm_heads x[4];
  int32_t n_x, heads, head_dim, tokens;   // heads of all tensors; tokens of a CTA
  FastDiv by_unit, by_heads, by_rest, by_pairs;
  const int32_t* positions;
  int64_t n_tokens;
  float sign;
};

template <typename T>
__device__ __forceinline__ void locate(const RopeLaunch& a, int64_t token, int head, const T** in, T** out) {
  int k = 0;
  while (k + 1 < a.n_x && head >= a.x[k].n_heads) head -= a.x[k++].n_heads;
  const kvprm_heads& x = a.x[k];
  *in = static_cast<const T*>(x.in) + token * x.in_token + head * x.in_head;
  *out = static_cast<T*>(x.out) + token * x.out_token + head * x.out_head;
}

// A unit is 16 bytes of pairs' first elements and the 16 bytes of their second ones (half layout), or
// 16 bytes of neighbouring pairs (interleaved); single pairs without VEC.
template <typename T, bool INTERLEAVED, bool VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeLaunch a) {
  extern __shared__ __align__(16) float s_rot[];
  const int pairs = a.tab.dim >> 1;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * a.tokens;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(a.tokens), a.n_tokens - first));
  float* s_cos = s_rot;
  float* s_sin = s_rot + a.tokens * pairs;
  fill_rotations(a.tab, a.by_pairs, a.positions, first, tokens, a.sign, s_cos, s_sin);
  __syncthreads();
  constexpr int kV = VEC ? 16 / sizeof(T) : (INTERLEAVED ? 2 : 1);   // elements of an access
  constexpr int kP = INTERLEAVED ? kV / 2 : kV;                      // pairs of a unit
  const uint32_t units = a.by_unit.d;                                // of a head
  const uint32_t total = static_cast<uint32_t>(tokens) * a.heads * units;
  for (uint32_t i = threadIdx.x; i < total; i += kThreads) {
    const uint32_t row = a.by_unit.div(i), u = i - row * units;
    const uint32_t t = a.by_heads.div(row), h = row - t * a.heads;
    const T* in;
    T* out;
    locate<T>(a, first + t, static_cast<int>(h), &in, &out);
    float cs[kP], sn[kP];
    const float *pc = s_cos + t * pairs + u * kP, *ps = s_sin + t * pairs + u * kP;
#pragma unroll
    for (int k = 0; k < kP; ++k) {
      cs[k] = pc[k];
      sn[k] = ps[k];
    }
    if constexpr (INTERLEAVED) {
      float x[kV], y[kV];
      load_n<T, kV, VEC>(in + u * kV, x);
#pragma unroll
      for (int k = 0; k < kP; ++k) {
        y[2 * k] = x[2 * k] * cs[k] - x[2 * k + 1] * sn[k];
        y[2 * k + 1] = x[2 * k + 1] * cs[k] + x[2 * k] * sn[k];
      }
      store_n<T, kV, VEC>(out + u * kV, y);
    } else {
      float x0[kV], x1[kV], y0[kV], y1[kV];
      load_n<T, kV, VEC>(in + u * kV, x0);
      load_n<T, kV, VEC>(in + pairs + u * kV, x1);
#pragma unroll
      for (int k = 0; k < kV; ++k) {
        y0[k] = x0[k] * cs[k] - x1[k] * sn[k];
        y1[k] = x1[k] * cs[k] + x0[k] * sn[k];
      }
      store_n<T, kV, VEC>(out + u * kV, y0);
      store_n<T, kV, VEC>(out + pairs + u * kV, y1);
    }
  }
  // the rest of each head passes unchanged
  constexpr int kR = VEC ? 16 / sizeof(T) : 1;
  const uint32_t rest = static_cast<uint32_t>(a.head_dim - a.tab.dim) / kR;
  if (rest == 0) return;
  for (uint32_t i = threadIdx.x; i < static_cast<uint32_t>(tokens) * a.heads * rest; i += kThreads) {
    const uint32_t row = a.by_rest.div(i), u = i - row * rest;
    const uint32_t t = a.by_heads.div(row), h = row - t * a.heads;
    const T* in;
    T* out;
    locate<T>(a, first + t, static_cast<int>(h), &in, &out);
    if (in == out) continue;
    if constexpr (VEC)
      reinterpret_cast<uint4*>(out + a.tab.dim)[u] = reinterpret_cast<const uint4*>(in + a.tab.dim)[u];
    else
      out[a.tab.dim + u] = in[a.tab.dim + u];
  }
}

// ---------------------------------------------------------------- cache write
struct WriteLaunch {
  RopeTable tab;           // dim 0: keys are not rotated
  const void *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  const int64_t* slots;
  const int32_t* positions;
  int64_t n_tokens, n_slots;
  uint8_t* pages;
  uint8_t* exponents;
  int32_t heads, head_dim, tokens;
  FastDiv by_rows, by_pairs;   // 2 * heads
};

// Eight elements from `i` on of a key row, rotated.  Partners outside the eight are read again (they
// are in L1: the row's other threads have just read them).
template <typename T, bool VEC>
__device__ __forceinline__ void rotate8(const RopeTable& tab, const float* cs, const float* sn, const T* row, int i,
                                        float (&x)[8]) {
  const int pairs = tab.dim >> 1;
  if (VEC && i >= tab.dim) return;   // a multiple of 8 elements is rotated
  if (tab.interleaved) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
      if (!VEC && i + k >= tab.dim) break;
      const float c = cs[(i + k) >> 1], s = sn[(i + k) >> 1], a = x[k], b = x[k + 1];
      x[k] = a * c - b * s;
      x[k + 1] = b * c + a * s;
    }
    return;
  }
  if constexpr (VEC) {   // a multiple of 8 pairs: the eight are all first or all second elements
    const bool second = i >= pairs;
    float y[8];
    load_n<T, 8, true>(row + (second ? i - pairs : i + pairs), y);
    const float *pc = cs + (second ? i - pairs : i), *ps = sn + (second ? i - pairs : i);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = x[k] * pc[k] + y[k] * (second ? ps[k] : -ps[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int e = i + k;
      if (e >= tab.dim) break;
      const bool second = e >= pairs;
      const int p = second ? e - pairs : e;
      const float y = to_f<T>(row[second ? p : e + pairs]);
      x[k] = x[k] * cs[p] + y * (second ? sn[p] : -sn[p]);
    }
  }
}

// The exponent of a row whose largest finite magnitude is `most`: the least e >= -127 with
// most <= 448 * 2^e = 1.75 * 2^(8 + e), from the number's own bits.
__device__ __forceinline__ int row_exponent(float most) {
  const uint32_t u = __float_as_uint(most);
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, -127);
}

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ uint2 e4m3_of8(const float (&x)[8], float f) {
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const __nv_fp8x2_storage_t a = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * k] * f, x[4 * k + 1] * f), __NV_SATFINITE, __NV_E4M3);
    const __nv_fp8x2_storage_t b = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * k + 2] * f, x[4 * k + 3] * f), __NV_SATFINITE, __NV_E4M3);
    w[k] = static_cast<uint32_t>(a) | (static_cast<uint32_t>(b) << 16);
  }
  return make_uint2(w[0], w[1]);
}

// head_dim / 16 threads per row: each takes eight elements of either half of the row, so that a
// rotated pair of the half layout meets in one thread, and the row's maximum in as many shuffles.
template <typename T, bool E4M3, bool VEC>
__global__ void __launch_bounds__(kThreads) write_kernel(const __grid_constant__ WriteLaunch a) {
  extern __shared__ __align__(16) float s_rot[];
  const int pairs = a.tab.dim >> 1;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * a.tokens;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(a.tokens), a.n_tokens - first));
  float* s_cos = s_rot;
  float* s_sin = s_rot + a.tokens * pairs;
  if (pairs > 0) {
    fill_rotations(a.tab, a.by_pairs, a.positions, first, tokens, 1.f, s_cos, s_sin);
    __syncthreads();
  }
  const int per_row = a.head_dim >> 4, half = a.head_dim >> 1, j = threadIdx.x & (per_row - 1);
  // A thread keeps its row of a token (its head's keys or values) and goes from token to token, as many tokens at a time
  // as the CTA's threads cover; a token of more rows than that takes several rounds.
  const int rows = 2 * a.heads, lane_row = threadIdx.x / per_row, at_once = kThreads / per_row;
  const int side = rows < at_once ? static_cast<int>(a.by_rows.div(lane_row)) : 0;   // which of the tokens at a time
  const int side_tokens = rows < at_once ? at_once / rows : 1;
  for (int r0 = 0; r0 < rows; r0 += at_once) {
    const int r = rows < at_once ? lane_row - side * rows : r0 + lane_row;
    const bool mine = r < rows && side < side_tokens;
    const bool kv = r >= a.heads;
    const int h = kv ? r - a.heads : r;
    const T* base = kv ? static_cast<const T*>(a.v) + h * a.v_head : static_cast<const T*>(a.k) + h * a.k_head;
    const int64_t token_step = kv ? a.v_token : a.k_token;
    for (int t0 = 0; t0 < tokens; t0 += side_tokens) {
      const int t = t0 + side;
      int64_t slot = -1;
      if (mine && t < tokens) slot = __ldg(a.slots + first + t);
      const bool live = slot >= 0 && slot < a.n_slots;
      float x0[8], x1[8];
      if (live) {
        const T* row = base + (first + t) * token_step;
        load_n<T, 8, VEC>(row + 8 * j, x0);
        load_n<T, 8, VEC>(row + half + 8 * j, x1);
        if (pairs > 0 && !kv) {
          const float *cs = s_cos + t * pairs, *sn = s_sin + t * pairs;
          if (!a.tab.interleaved && pairs == half) {
            float c[8], s[8];
            load_n<float, 8, true>(cs + 8 * j, c);
            load_n<float, 8, true>(sn + 8 * j, s);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float p = x0[k], q = x1[k];
              x0[k] = p * c[k] - q * s[k];
              x1[k] = q * c[k] + p * s[k];
            }
          } else {
            rotate8<T, VEC>(a.tab, cs, sn, row, 8 * j, x0);
            rotate8<T, VEC>(a.tab, cs, sn, row, half + 8 * j, x1);
          }
        }
      }
      const int64_t out_row = ((slot >> 4) * rows + r) * 16 + (slot & 15);   // (rows of a page: keys' heads, then values')
      if constexpr (E4M3) {
        // the largest magnitude, NaN if there is one
        float most = 0.f;
        if (live) {
#pragma unroll
          for (int k = 0; k < 8; ++k) most = max_nan(most, max_nan(fabsf(x0[k]), fabsf(x1[k])));
        }
        for (int off = per_row >> 1; off > 0; off >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, off));
        const bool nan = most != most;
        if (__any_sync(0xffffffffu, most == INFINITY)) {   // the largest finite one, then
          float finite = 0.f;
          if (live) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float p = fabsf(x0[k]), q = fabsf(x1[k]);
              finite = fmaxf(finite, fmaxf(p < INFINITY ? p : 0.f, q < INFINITY ? q : 0.f));
            }
          }
          for (int off = per_row >> 1; off > 0; off >>= 1) finite = fmaxf(finite, __shfl_xor_sync(0xffffffffu, finite, off));
          most = finite;
        }
        if (!live) continue;
        const int e = nan ? 0 : row_exponent(most);
        const float f = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);   // 2^-e, e in [-127, 120]
        uint8_t* out = a.pages + out_row * a.head_dim;
        *reinterpret_cast<uint2*>(out + 8 * j) = e4m3_of8(x0, f);
        *reinterpret_cast<uint2*>(out + half + 8 * j) = e4m3_of8(x1, f);
        if (j == 0) a.exponents[out_row] = nan ? 255 : static_cast<uint8_t>(e + 127);
      } else {
        if (!live) continue;
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.pages) + out_row * a.head_dim;
        store_n<__nv_bfloat16, 8, true>(out + 8 * j, x0);
        store_n<__nv_bfloat16, 8, true>(out + half + 8 * j, x1);
      }
    }
  }
}

// ---------------------------------------------------------------- expand
// Pieces of 8 codes: an 8-byte load, the row's power of two, a 16-byte store, so that a warp's stores are 512 bytes side by
// side (with 16 codes a thread each store left every other 16 bytes out: 86 % of the copy rate).
constexpr int kExpandPer = 4;   // pieces of a thread
__global__ void __launch_bounds__(kThreads) expand_kernel(const uint2* __restrict__ pages,
                                                          const uint8_t* __restrict__ exponents,
                                                          const int32_t* __restrict__ src,
                                                          const int32_t* __restrict__ dst, int64_t n_pages,
                                                          int64_t out_pages, int rows, int row_shift,
                                                          uint4* __restrict__ out) {
  const int64_t s = __ldg(src + blockIdx.x), d = __ldg(dst + blockIdx.x);
  if (s < 0 || s >= n_pages || d < 0 || d >= out_pages) return;
  const int pieces = rows << row_shift;   // of a page
  const int p0 = blockIdx.y * (kThreads * kExpandPer) + threadIdx.x;
  uint2 c[kExpandPer];
  float f[kExpandPer];
#pragma unroll
  for (int i = 0; i < kExpandPer; ++i) {
    const int p = p0 + i * kThreads;
    if (p >= pieces) continue;
    c[i] = __ldg(pages + s * pieces + p);
    f[i] = row_factor(__ldg(exponents + s * rows + (p >> row_shift)));
  }
#pragma unroll
  for (int i = 0; i < kExpandPer; ++i) {
    const int p = p0 + i * kThreads;
    if (p >= pieces) continue;
    uint32_t r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __half2_raw h2 = __nv_cvt_fp8x2_to_halfraw2(
          static_cast<__nv_fp8x2_storage_t>((k < 2 ? c[i].x : c[i].y) >> (16 * (k & 1))), __NV_E4M3);
      const float2 v = __half22float2(__half2(h2));
      r[k] = pack_bf16(v.x * f[i], v.y * f[i]);
    }
    out[d * pieces + p] = make_uint4(r[0], r[1], r[2], r[3]);
  }
}

// ---------------------------------------------------------------- host
int size_of(int32_t dtype) { return dtype == KVPRM_F32 ? 4 : dtype == KVPRM_BF16 || dtype == KVPRM_F16 ? 2 : 0; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return n;
}

// Tokens of a CTA: one while there are fewer than four CTAs per SM, so that a step's few tokens spread
// over the SMs; then up to `most`, which share a launch's fixed costs.
int tokens_per_cta(int64_t n, int sms, int most) {
  const int64_t t = n / (4 * static_cast<int64_t>(sms));
  return static_cast<int>(t < 1 ? 1 : t > most ? most : t);
}

template <typename K, typename A>
int launch(K kernel, dim3 grid, size_t smem, const A& args, void* stream, const char* what) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args);
  if (e != cudaSuccess) return operator_fail(KVPRM_ECUDA, "%s: %s", what, cudaGetErrorString(e));
  return KVPRM_OK;
}

template <typename T>
int launch_rope(const RopeLaunch& a, bool vec, unsigned grid, void* stream) {
  const size_t smem = static_cast<size_t>(a.tokens) * a.tab.dim * sizeof(float);
  auto k = a.tab.interleaved ? (vec ? rope_kernel<T, true, true> : rope_kernel<T, true, false>)
                             : (vec ? rope_kernel<T, false, true> : rope_kernel<T, false, false>);
  return launch(k, dim3(grid), smem, a, stream, "rotary launch");
}

template <typename T>
int launch_write(const WriteLaunch& a, bool e4m3, bool vec, unsigned grid, void* stream) {
  const size_t smem = static_cast<size_t>(a.tokens) * a.tab.dim * sizeof(float);
  auto k = e4m3 ? (vec ? write_kernel<T, true, true> : write_kernel<T, true, false>)
                : (vec ? write_kernel<T, false, true> : write_kernel<T, false, false>);
  return launch(k, dim3(grid), smem, a, stream, "cache write launch");
}

}  // namespace

int check_cache(const kvprm_cache* c, const char* who) {
  if (!c) return operator_fail(KVPRM_EINVAL, "%s: no cache", who);
  if (c->format != KVPRM_CACHE_BF16 && c->format != KVPRM_CACHE_E4M3)
    return operator_fail(KVPRM_EINVAL, "%s: cache format %d", who, c->format);
  if (c->head_dim != 64 && c->head_dim != 128)
    return operator_fail(KVPRM_EINVAL, "%s: head_dim %d is not 64 or 128", who, c->head_dim);
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_pages < 0 || c->n_pages > (int64_t{1} << 30))
    return operator_fail(KVPRM_EINVAL, "%s: n_kv_heads %d, n_pages %lld", who, c->n_kv_heads,
                         static_cast<long long>(c->n_pages));
  if ((c->n_pages > 0 && !c->pages) || !aligned16(c->pages))
    return operator_fail(KVPRM_EINVAL, "%s: pages are NULL or not 16-byte aligned", who);
  if (c->format == KVPRM_CACHE_E4M3 && ((c->n_pages > 0 && !c->exponents) || !aligned16(c->exponents)))
    return operator_fail(KVPRM_EINVAL, "%s: exponents are NULL or not 16-byte aligned", who);
  return KVPRM_OK;
}

}  // namespace kvprm

using namespace kvprm;

extern "C" {

const char* kvprm_operator_error(void) { return g_message; }

int kvprm_rope_create(const kvprm_rope_config* c, kvprm_rope** out) {
  if (!out) return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: out is NULL");
  *out = nullptr;
  if (!c) return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: no config");
  const int rd = c->rotary_dim;
  if (rd < 2 || rd > 2 * kMaxPairs || rd % 2 != 0)
    return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: rotary_dim %d is not an even number in 2 .. %d", rd, 2 * kMaxPairs);
  if (c->interleaved != 0 && c->interleaved != 1)
    return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: interleaved %d", c->interleaved);
  if (c->scaling < KVPRM_ROPE_NONE || c->scaling > KVPRM_ROPE_SMOOTH)
    return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: scaling %d", c->scaling);
  if (!(c->base > 1.0) || !std::isfinite(c->base) || !std::isfinite(static_cast<float>(c->magnitude)))
    return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: base %g, magnitude %g", c->base, c->magnitude);
  if (c->scaling != KVPRM_ROPE_NONE && (!(c->factor >= 1.0) || !std::isfinite(c->factor)))
    return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: factor %g", c->factor);
  if (c->scaling == KVPRM_ROPE_BASE && rd == 2)
    return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: a stretched base needs rotary_dim > 2");
  const bool turns_matter = c->scaling == KVPRM_ROPE_RAMP || c->scaling == KVPRM_ROPE_SMOOTH;
  if (turns_matter && (c->original_len < 1 || !(c->low > 0.0) || !(c->high > c->low) || !std::isfinite(c->high)))
    return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: original_len %d, low %g, high %g", c->original_len, c->low, c->high);
  double base = c->base;
  if (c->scaling == KVPRM_ROPE_BASE) base *= std::pow(c->factor, static_cast<double>(rd) / (rd - 2));
  if (!std::isfinite(base)) return operator_fail(KVPRM_EINVAL, "kvprm_rope_create: base %g times factor %g", c->base, c->factor);
  kvprm_rope* r = new (std::nothrow) kvprm_rope();
  if (!r) return operator_fail(KVPRM_ENOMEM, "kvprm_rope_create: out of memory");
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  double first = 0.0, last = 0.0;   // RAMP: the pairs between which the weight falls
  if (c->scaling == KVPRM_ROPE_RAMP) {
    auto pair_at = [&](double n) { return rd * std::log(c->original_len / (kTwoPi * n)) / (2.0 * std::log(base)); };
    first = std::fmax(0.0, std::floor(pair_at(c->high)));
    last = std::fmin(rd - 1.0, std::ceil(pair_at(c->low)));
  }
  for (int i = 0; i < rd / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rd);
    double kept = 1.0;   // weight of the unstretched frequency
    if (c->scaling == KVPRM_ROPE_LINEAR) kept = 0.0;
    if (c->scaling == KVPRM_ROPE_RAMP) kept = 1.0 - (i - first) / std::fmax(last - first, 1e-3);
    if (c->scaling == KVPRM_ROPE_SMOOTH) kept = (c->original_len * f / kTwoPi - c->low) / (c->high - c->low);
    kept = std::fmin(1.0, std::fmax(0.0, kept));
    double turn = f / kTwoPi;
    if (c->scaling == KVPRM_ROPE_LINEAR || turns_matter) turn = kept * turn + (1.0 - kept) * (turn / c->factor);
    // below one turn (base > 1, so f <= 1): 2^64 turn fits, its last bits those of the 53-bit product
    r->table.turns[i] = static_cast<uint64_t>(std::rint(std::ldexp(turn, 64)));
  }
  r->table.magnitude = static_cast<float>(c->magnitude);
  r->table.dim = rd;
  r->table.interleaved = c->interleaved;
  *out = r;
  return KVPRM_OK;
}

void kvprm_rope_destroy(kvprm_rope* rope) { delete rope; }

int kvprm_rope_turns(const kvprm_rope* rope, uint64_t* turns) {
  if (!rope || !turns) return operator_fail(KVPRM_EINVAL, "kvprm_rope_turns: NULL argument");
  for (int i = 0; i < rope->table.dim / 2; ++i) turns[i] = rope->table.turns[i];
  return KVPRM_OK;
}

int kvprm_rope_rotate(const kvprm_rope* rope, int32_t dtype, int32_t head_dim, const int32_t* positions,
                      int64_t n_tokens, int32_t inverse, const kvprm_heads* x, int32_t n_x, void* stream) {
  const char* who = "kvprm_rope_rotate";
  const int size = size_of(dtype);
  if (!rope || !x || n_x < 1 || n_x > 4) return operator_fail(KVPRM_EINVAL, "%s: no rope, or %d tensors (1 .. 4)", who, n_x);
  if (size == 0) return operator_fail(KVPRM_EINVAL, "%s: dtype %d", who, dtype);
  if (head_dim < rope->table.dim || head_dim > kMaxHeadDim)
    return operator_fail(KVPRM_EINVAL, "%s: head_dim %d, %d of it rotated (at most 512)", who, head_dim, rope->table.dim);
  if (inverse != 0 && inverse != 1) return operator_fail(KVPRM_EINVAL, "%s: inverse %d", who, inverse);
  if (n_tokens < 0) return operator_fail(KVPRM_EINVAL, "%s: n_tokens %lld", who, static_cast<long long>(n_tokens));
  RopeLaunch a;
  a.tab = rope->table;
  a.heads = 0;
  const int per = 16 / size, dim = a.tab.dim;
  bool vec = head_dim % per == 0 && (a.tab.interleaved ? dim : dim / 2) % per == 0;
  for (int k = 0; k < n_x; ++k) {
    if (x[k].n_heads < 0 || x[k].n_heads > kMaxHeads - a.heads)
      return operator_fail(KVPRM_EINVAL, "%s: %d heads (at most 1024 in all)", who, x[k].n_heads);
    if (n_tokens > 0 && x[k].n_heads > 0 && (!x[k].in || !x[k].out)) return operator_fail(KVPRM_EINVAL, "%s: tensor %d is NULL", who, k);
    if ((reinterpret_cast<uintptr_t>(x[k].in) | reinterpret_cast<uintptr_t>(x[k].out)) % size)
      return operator_fail(KVPRM_EINVAL, "%s: tensor %d is not aligned to its elements", who, k);
    a.x[k] = x[k];
    a.heads += x[k].n_heads;
    vec = vec && aligned16(x[k].in) && aligned16(x[k].out) &&
          ((x[k].in_token | x[k].in_head | x[k].out_token | x[k].out_head) * size) % 16 == 0;
  }
  if (n_tokens == 0 || a.heads == 0) return KVPRM_OK;
  if (!positions) return operator_fail(KVPRM_EINVAL, "%s: positions are NULL", who);
  const int sms = sm_count();
  if (sms == 0) return operator_fail(KVPRM_ECUDA, "%s: no device", who);
  a.n_x = n_x;
  a.head_dim = head_dim;
  a.tokens = tokens_per_cta(n_tokens, sms, kRopeTokens);
  const int64_t grid = (n_tokens + a.tokens - 1) / a.tokens;
  if (grid > 0x7FFFFFFF) return operator_fail(KVPRM_EINVAL, "%s: n_tokens %lld", who, static_cast<long long>(n_tokens));
  a.by_unit = FastDiv(static_cast<uint32_t>(vec ? (a.tab.interleaved ? dim : dim / 2) / per : dim / 2));
  a.by_heads = FastDiv(static_cast<uint32_t>(a.heads));
  a.by_pairs = FastDiv(static_cast<uint32_t>(dim / 2));
  a.by_rest = FastDiv(static_cast<uint32_t>(head_dim > dim ? (head_dim - dim) / (vec ? per : 1) : 1));
  a.positions = positions;
  a.n_tokens = n_tokens;
  a.sign = inverse ? -1.f : 1.f;
  const unsigned g = static_cast<unsigned>(grid);
  if (dtype == KVPRM_F32) return launch_rope<float>(a, vec, g, stream);
  if (dtype == KVPRM_BF16) return launch_rope<__nv_bfloat16>(a, vec, g, stream);
  return launch_rope<__half>(a, vec, g, stream);
}

int kvprm_cache_write(const kvprm_cache* cache, int32_t dtype, const void* k, int64_t k_token, int64_t k_head,
                      const void* v, int64_t v_token, int64_t v_head, const int64_t* slots, int64_t n_tokens,
                      const kvprm_rope* rope, const int32_t* positions, void* stream) {
  const char* who = "kvprm_cache_write";
  if (const int rc = check_cache(cache, who)) return rc;
  const int size = size_of(dtype);
  if (size == 0) return operator_fail(KVPRM_EINVAL, "%s: dtype %d", who, dtype);
  if (n_tokens < 0) return operator_fail(KVPRM_EINVAL, "%s: n_tokens %lld", who, static_cast<long long>(n_tokens));
  if (rope && rope->table.dim > cache->head_dim)
    return operator_fail(KVPRM_EINVAL, "%s: %d elements rotated of head_dim %d", who, rope->table.dim, cache->head_dim);
  if (n_tokens == 0) return KVPRM_OK;
  if ((rope == nullptr) != (positions == nullptr))
    return operator_fail(KVPRM_EINVAL, "%s: rope and positions come together", who);
  if (!k || !v || !slots) return operator_fail(KVPRM_EINVAL, "%s: k, v or slots are NULL", who);
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % size || reinterpret_cast<uintptr_t>(slots) % 8)
    return operator_fail(KVPRM_EINVAL, "%s: k, v or slots are not aligned to their elements", who);
  const int sms = sm_count();
  if (sms == 0) return operator_fail(KVPRM_ECUDA, "%s: no device", who);
  WriteLaunch a;
  if (rope)
    a.tab = rope->table;
  else
    a.tab.dim = a.tab.interleaved = 0;
  bool vec = aligned16(k) && aligned16(v) && ((k_token | k_head | v_token | v_head) * size) % 16 == 0;
  vec = vec && (a.tab.interleaved ? a.tab.dim : a.tab.dim / 2) % 8 == 0;
  a.k = k;
  a.v = v;
  a.k_token = k_token;
  a.k_head = k_head;
  a.v_token = v_token;
  a.v_head = v_head;
  a.slots = slots;
  a.positions = positions;
  a.n_tokens = n_tokens;
  a.n_slots = cache->n_pages * 16;
  a.pages = static_cast<uint8_t*>(cache->pages);
  a.exponents = static_cast<uint8_t*>(cache->exponents);
  a.heads = cache->n_kv_heads;
  a.head_dim = cache->head_dim;
  a.tokens = tokens_per_cta(n_tokens, sms, kWriteTokens);
  a.by_rows = FastDiv(static_cast<uint32_t>(2 * a.heads));
  a.by_pairs = FastDiv(static_cast<uint32_t>(a.tab.dim > 0 ? a.tab.dim / 2 : 1));
  const int64_t grid = (n_tokens + a.tokens - 1) / a.tokens;
  if (grid > 0x7FFFFFFF) return operator_fail(KVPRM_EINVAL, "%s: n_tokens %lld", who, static_cast<long long>(n_tokens));
  const unsigned g = static_cast<unsigned>(grid);
  const bool e4m3 = cache->format == KVPRM_CACHE_E4M3;
  if (dtype == KVPRM_F32) return launch_write<float>(a, e4m3, vec, g, stream);
  if (dtype == KVPRM_BF16) return launch_write<__nv_bfloat16>(a, e4m3, vec, g, stream);
  return launch_write<__half>(a, e4m3, vec, g, stream);
}

int kvprm_cache_expand(const kvprm_cache* cache, const int32_t* src, const int32_t* dst, int64_t n, void* out,
                       int64_t out_pages, void* stream) {
  const char* who = "kvprm_cache_expand";
  if (const int rc = check_cache(cache, who)) return rc;
  if (cache->format != KVPRM_CACHE_E4M3) return operator_fail(KVPRM_EINVAL, "%s: the cache is not quantised", who);
  if (n < 0 || n > 0x7FFFFFFF || out_pages < 0) return operator_fail(KVPRM_EINVAL, "%s: n %lld, out_pages %lld", who, static_cast<long long>(n), static_cast<long long>(out_pages));
  if (n == 0 || cache->n_pages == 0 || out_pages == 0) return KVPRM_OK;
  if (!src || !dst || !out || !aligned16(out)) return operator_fail(KVPRM_EINVAL, "%s: src, dst or out are NULL, or out is not 16-byte aligned", who);
  const int rows = 2 * cache->n_kv_heads * 16, shift = cache->head_dim == 128 ? 4 : 3;
  const int pieces = rows << shift;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(n), static_cast<unsigned>((pieces + kThreads * kExpandPer - 1) / (kThreads * kExpandPer)), 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = static_cast<cudaStream_t>(stream);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, expand_kernel, static_cast<const uint2*>(cache->pages),
                                           static_cast<const uint8_t*>(cache->exponents), src, dst, cache->n_pages,
                                           out_pages, rows, shift, static_cast<uint4*>(out));
  if (e != cudaSuccess) return operator_fail(KVPRM_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  return KVPRM_OK;
}

}  // extern "C"
