// The rotary table as kernels take it (internal): the handle's host copy, passed by value.
#pragma once

#include <stdint.h>

#include "../../include/kvprm.h"

namespace kvprm {

constexpr int kMaxPairs = 128;

struct RopeTable {
  uint64_t turns[kMaxPairs];   // of pair i per position, in units of 2^-64
  float magnitude;
  int32_t dim;                 // rotated elements of a head, 2 * pairs
  int32_t interleaved;
};

#ifdef __CUDACC__
// A row's power of two from its exponent byte: 2^(e - 127), a subnormal at 0, NaN at 255.
__device__ __forceinline__ float row_factor(uint32_t e) {
  return __uint_as_float((e << 23) | (((e + 1u) & 0xFEu) == 0u ? 0x400000u : 0u));
}
// Eight e2m1 codes of a word as fp16 pairs, in their order (exact, an instruction a pair).
__device__ __forceinline__ void f16_of_e2m1(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
#endif

// Argument checks that the cache's entry points share.
int check_cache(const kvprm_cache* c, const char* who);

// Records the calling thread's message of a failed operator call; returns code.
int operator_fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace kvprm

struct kvprm_rope {
  kvprm::RopeTable table;
};
