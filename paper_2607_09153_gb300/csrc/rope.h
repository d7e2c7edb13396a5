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
#endif

// Argument checks that the cache's entry points share.
int check_cache(const kvprm_cache* c, const char* who);

// Records the calling thread's message of a failed operator call; returns code.
int operator_fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace kvprm

struct kvprm_rope {
  kvprm::RopeTable table;
};
