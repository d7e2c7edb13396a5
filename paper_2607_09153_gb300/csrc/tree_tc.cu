// Attention of drafted tokens over the paged cache on the tensor cores (tcgen05), for more than 32 query
// rows (drafted token and head of the kv head's group) per sequence and kv head.
//
// A pair (tree.h) is one kv head of a sequence and one or two tiles of 128 query rows; its keys come in
// chunks of 128 (8 pages).  For each chunk and tile ("unit"): S = Q K^T into tensor memory, a softmax step
// per row by one thread, the weights back over S as bf16, O += P V from there.  Two softmax groups of 128
// threads work on alternate units with an S buffer and an O accumulator each: the two tiles of a pair, which
// then share each chunk's keys and values, or, where the pair has one tile, its even and odd chunks as two
// streams that meet at the end.  Either way one group's softmax runs beside the other's matrix products, and
// the groups never wait for each other within a part.
//   warps 0-3, 4-7   softmax groups (thread = row = lane of tensor memory)
//   warps 8-15       producers: Q tiles, drafted tokens' keys and values, and with an 8-bit cache every chunk,
//                    converted to bf16 (exact: a power of two per row changes no mantissa)
//   warp 16          TMA: bf16 pages straight into the tiles
//   warp 17          issues every MMA, in an order that keeps one unit's S ahead of the other's O
//
// What bounds it, measured on a GB300.  Two tiles: a group's chain of S (800 cycles: its operands take all of
// shared memory's bandwidth), softmax (1,500) and O (500), 3,400 cycles a chunk for both groups: 8 kv heads, 64
// tokens of 4 heads each over 4 x 16,384 bf16 tokens in 80 us, 860 TFLOP/s.  An 8-bit chunk: its conversion, some
// 1,800 cycles of the eight producer warps for a tile of 128 x 128, which beside two tiles' products takes
// 2,800: 16 sequences of 4 heads with 126 rows over 9,001 tokens in 86 us (bf16: 70).  Short calls: what a part
// begins and ends with, 5 and 2 us, and the join.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "ptx.cuh"
#include "rope.h"
#include "tree.h"

namespace kvprm {

namespace {

constexpr int kThreads = 576;
constexpr int kRows = TreeTc::ROWS, kChunk = TreeTc::BLOCK, kPages = kChunk / kTreePage;
constexpr int kProducers = 256;
constexpr int kWarpTma = 16, kWarpMma = 17;
constexpr float kMargin = 8.f;   // log2 units that scores may pass a running maximum by
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;   // S buffers at 0 and 128, accumulators at 256 and 384
constexpr int kFlagSets = 8;     // parts whose marks may be in flight (a ring of eight slots reaches five parts ahead)

template <int HD, bool E4M3>
struct Smem {
  static constexpr uint32_t kTile = kChunk * HD * 2;             // one chunk's keys or values, or one tile of Q
  static constexpr int kSlots = HD == 128 ? (E4M3 ? 3 : 4) : 8;
  static constexpr uint32_t kQ = 0;                              // two tiles
  static constexpr uint32_t kSlot0 = kQ + 2 * kTile;
  static constexpr uint32_t kMl = kSlot0 + kSlots * kTile;   // float2 [2][128]
  static constexpr uint32_t kEnd = kMl + 2 * kRows * 8;
  static constexpr size_t kDynamic = kEnd + 1024;
};

struct Static {   // in static shared memory
  int32_t off[kTreeSeqs + 1];
  int32_t sum[kThreads / 32];
  uint64_t slot_full[8], slot_empty[8];
  uint64_t draft_go[8];   // bf16 cache: a free slot that is the producers' to fill
  uint64_t q_full, q_empty, s_full[2], p_full[2], part_done, o_free;
  uint32_t bad_drafts[kFlagSets][32];   // drafted tokens of a part whose values are not finite
  int bad[kFlagSets];                   // of a part: a page outside the cache, a bad draft (1, 2)
  uint32_t tmem;
  TreePart part[8];                     // of the softmax warps, and where they are on the line (in registers the two made
  int4 walk[8];                         // the loop over chunks spill)
  int err;   // a wait gave up (after which the CTA's other waits are short, and its rows NaN)
};

// The items of a part: its chunks' keys and values, in the order in which the matrix products take them.  Keys and
// values in turn where two tiles share a chunk; keys one chunk further ahead where the chunks alternate between the
// groups (K0 K1 V0 K2 V1 ..): the S that follows an O is then two chunks on, and no slot holds values that wait for
// their softmax while keys are needed.
struct Items {
  int tiles, n;   // n: two per chunk
  __device__ __forceinline__ explicit Items(const TreePart& p) : tiles(p.tiles), n(2 * (p.c1 - p.c0)) {}
  __device__ __forceinline__ int keys(int c) const { return tiles == 2 ? 2 * c : c == 0 ? 0 : 2 * c - 1; }
  __device__ __forceinline__ int values(int c) const { return tiles == 2 || 2 * c == n - 2 ? 2 * c + 1 : 2 * c + 2; }
  // the chunk of an item, and whether it is its values
  __device__ __forceinline__ int chunk(int item, int* kv) const {
    const bool last = item == n - 1;
    *kv = tiles == 2 ? item & 1 : last || (item > 0 && (item & 1) == 0);
    return tiles == 2 || last ? item >> 1 : *kv ? (item >> 1) - 1 : (item + 1) >> 1;
  }
};

// Tiles in shared memory, 128 rows of HD columns: [8-row group][64-column part][8 rows][128 bytes] under the 128-byte
// swizzle, a K-major operand (Q, keys) and an MN-major one (values) alike, and what one TMA box per page leaves.  (With
// [part][128 rows] a page took a box per part, and at about 120 cycles a box the TMA unit, not memory, bounded the call;
// with [page][part][16 rows] S took twice the instructions of half the columns, and they bounded it.)
constexpr uint32_t kAtom = 1024;   // eight rows of a part
template <int HD>
__device__ __forceinline__ uint32_t swizzled(int row, int piece) {   // of a 16-byte piece of a row
  return static_cast<uint32_t>(row >> 3) * (HD * 16) + static_cast<uint32_t>(piece >> 3) * kAtom + (row & 7) * 128 +
         (((piece & 7) ^ (row & 7)) << 4);
}

// mbar_wait (ptx.cuh) with the barrier's own suspension: most of this kernel's warps wait most of the time, and share
// their schedulers with the softmax.
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, int* err) {
  const uint32_t at = smem_u32(bar);
  if (mbar_try_wait(at, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  for (;;) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(at), "r"(parity), "r"(20000u)   // ns
        : "memory");
    if (ok) return true;
    const uint64_t dt = global_timer_ns() - t0;
    if (dt < kErrPollNs) continue;
    if (*(volatile int*)err != 0) return false;
    if (dt > kWaitTimeoutNs) {
      atomicCAS(err, 0, kDevTimeout);
      return false;
    }
  }
}

__device__ __forceinline__ uint4 ldg_stream(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// As tmem_st16 (ptx.cuh), 8 columns.
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
               "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
               "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
               : "memory");
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return r;
}
// A product's steps are issued by one lane in a branch of its own, with descriptors at fixed steps from a base: some ten
// instructions a step.  (With the warp converged, an elected lane per step, each took forty.)
__device__ __forceinline__ bool elect_lane() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// Sixteen e4m3 codes as bf16 times a row's power of two.  A code's exponent and mantissa at bf16's place are 2^-120 of its
// value; f1 (times f2, where the two do not fit one factor) is 2^120 times the row's power.  The even and the odd codes of
// a word each become a pair, so that the head's dimensions come in the order 0 2 1 3, 4 6 5 7 ..: Q and the drafted
// tokens are laid out alike (paired), and the outputs are put back in order.
//   bf16 has no place for the NaN codes, 0x7F and 0xFF: there they would be 480.  So where a page has one, or a row that needs
// two factors, it takes the longer form (not PLAIN); a factor of zero, a row past the length, keeps NaN out.
template <bool PLAIN>
__device__ __forceinline__ void bf16_of16(const uint4& c, uint32_t f1, uint32_t f2, uint4* lo, uint4* hi) {
  auto pair = [&](uint32_t w, uint32_t* e, uint32_t* o) {
    const uint32_t even = (w << 4) & 0x07F007F0u, odd = (w >> 4) & 0x07F007F0u;
    *e = mul_bf16x2(even | ((w << 8) & 0x80008000u), f1);
    *o = mul_bf16x2(odd | (w & 0x80008000u), f1);
    if (PLAIN) return;
    auto nans = [&](uint32_t v) {
      return f1 == 0u ? 0u : ((v & 0xFFFFu) == 0x07F0u ? 0x7FC0u : 0u) | (v >> 16 == 0x07F0u ? 0x7FC00000u : 0u);
    };
    *e = mul_bf16x2(*e, f2) | nans(even);
    *o = mul_bf16x2(*o, f2) | nans(odd);
  };
  pair(c.x, &lo->x, &lo->y);
  pair(c.y, &lo->z, &lo->w);
  pair(c.z, &hi->x, &hi->y);
  pair(c.w, &hi->z, &hi->w);
}
// Bit 7 of a byte is set in the result where w's byte is a NaN code, and there is no such bit where none is: a carry into it,
// or out of the byte below, comes of seven ones alone.
__device__ __forceinline__ uint32_t nan_carries(uint32_t w) { return (w + 0x01010101u) ^ w; }
__device__ __forceinline__ uint4 paired(const uint4& v) {
  return make_uint4(__byte_perm(v.x, v.y, 0x5410), __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x5410),
                    __byte_perm(v.z, v.w, 0x7632));
}
template <int N>
__device__ __forceinline__ void in_order(float (&o)[N]) {
#pragma unroll
  for (int i = 1; i < N; i += 4) {
    const float x = o[i];
    o[i] = o[i + 1];
    o[i + 1] = x;
  }
}

// (a bound of 640 threads: 96 registers, what five warps of a scheduler can have)
template <int HD, bool E4M3>
__global__ void __launch_bounds__(640, 1) tree_tc_kernel(const __grid_constant__ TreeLaunch a,
                                                         const __grid_constant__ CUtensorMap map) {
  using SM = Smem<HD, E4M3>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Static st;
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t{1023});
  int* err = &st.err;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 8; ++i) {
      mbar_init(&st.slot_full[i], E4M3 ? kProducers / 32 : 1);
      mbar_init(&st.slot_empty[i], 1);
      mbar_init(&st.draft_go[i], 1);
    }
    mbar_init(&st.q_full, 1);
    mbar_init(&st.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&st.s_full[i], 1);
      mbar_init(&st.p_full[i], 4);
    }
    st.err = 0;
    mbar_init(&st.part_done, 1);
    mbar_init(&st.o_free, 8);
    fence_mbar_init();
    if constexpr (!E4M3) tma_prefetch_desc(&map);
  }
  if (threadIdx.x < kFlagSets * 32) st.bad_drafts[threadIdx.x >> 5][lane] = 0;
  if (threadIdx.x < kFlagSets) st.bad[threadIdx.x] = 0;
  if (warp == kWarpMma) {
    tmem_alloc(&st.tmem, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  grid_dep_launch();
  tree_line<TreeTc, kThreads, HD>(a, st.off, st.sum);   // barriers inside
  tc_fence_after();
  const uint32_t tmem = st.tmem;
  const int32_t total = st.off[a.n_seqs];
  const TreeShares shares(total, gridDim.x, a.weight_full);
  tree_leave_line(a, st.off, shares.ctas);
  const int me = blockIdx.x;
  const bool idle = me >= shares.ctas || total == 0;
  int32_t u = idle ? 0 : shares.begin(me);
  int32_t u_end = idle ? 0 : shares.begin(me + 1);
  int s = idle ? 0 : tree_find(st.off, a.n_seqs, u);
  TreePart p;
  auto next_part = [&]() { return tree_next<TreeTc>(a, st.off, u, u_end, s, p); };

  if (warp == kWarpTma) {
    // ------------------------------------------------ TMA
    const uint64_t pol = policy_evict_normal();
    uint32_t n = 0;   // items of earlier parts
    bool ok = true;
    auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_for(bar, parity, err)); };
    for (int part = 0; !E4M3 && ok && next_part(); ++part) {
      const int32_t* table = a.t.block_table + static_cast<int64_t>(a.seq0 + p.s) * a.t.max_blocks;
      const int pages = (p.q.len + kTreePage - 1) / kTreePage;
      const Items items(p);
      // page ids of four chunks, a page per lane, and of the next four (loaded long before they are needed); -1: no page
      // there, -2: not a page of the cache
      auto ids_of = [&](int four) {
        const int at = four * 32 + lane;
        if (at >= pages) return -1;
        const int32_t page = __ldg(table + at);
        return page < 0 || page >= a.n_pages ? -2 : page;
      };
      int four = p.c0 >> 2;
      int32_t ids = ids_of(four), ids_next = ids_of(four + 1);
      for (int item = 0; item < items.n && ok; ++item) {
        int kv;
        const int c = p.c0 + items.chunk(item, &kv);
        const bool cached = c < p.q.cached_blocks;
        if (kv && (c >> 2) > four) {   // (keys are at most a chunk ahead of values)
          ++four;
          ids = ids_next;
          ids_next = ids_of(four + 1);
        }
        int32_t id[kPages];
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kPages; ++i) {
          id[i] = __shfl_sync(0xffffffffu, (c >> 2) > four ? ids_next : ids, (c & 3) * kPages + i);
          bad = bad || id[i] == -2;
        }
        // This warp waits for every use of a slot, also where the producers fill it: a wait by parity sees only
        // the phase before the present one, so none may be left out.
        const uint32_t i = n + item, slot = i % SM::kSlots;
        if (i >= SM::kSlots) ok = wait_all(&st.slot_empty[slot], (i / SM::kSlots - 1) & 1u);
        if (!ok || lane != 0) continue;
        if (!cached) {
          mbar_arrive(&st.draft_go[slot]);
          continue;
        }
        // (a part's marks are set once a slot of it is free: no earlier part then holds the same set)
        if (bad) atomicOr(&st.bad[part % kFlagSets], 1);
        mbar_arrive_expect_tx(&st.slot_full[slot], SM::kTile);
        // a box is a page's rows of one head; a place without a page reads one that does not exist and arrives as zeros
        uint8_t* dst = base + SM::kSlot0 + slot * SM::kTile;
#pragma unroll
        for (int k = 0; k < kPages; ++k)
          tma_load_5d(dst + k * (HD * 32), &map, &st.slot_full[slot], 0, 0, 0, 0,
                      id[k] >= 0 ? (2 * id[k] + kv) * a.n_kv + p.g : -1, pol);
      }
      n += items.n;
    }
    // Nothing of this warp's is in flight when the CTA ends: the matrix products waited for every load.  After a wait
    // that gave up, a millisecond is far beyond a load's time.
    if (!ok) {
      const uint64_t t0 = global_timer_ns();
      while (global_timer_ns() - t0 < 1000000ull) __nanosleep(1000);
    }
  } else if (warp == kWarpMma) {
    // ------------------------------------------------ MMA
    const uint32_t id_s = idesc_bf16_f32(kRows, kChunk), id_o = idesc_bf16_f32(kRows, HD) | kIdescMnMajorB;
    auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_for(bar, parity, err)); };
    uint32_t n = 0, phase = 0;   // phase: per group, the parity of its next p_full
    bool ok = true;
    for (int part = 0; next_part(); ++part) {
      const Items items(p);
      const int units = (p.c1 - p.c0) * p.tiles;
      if (!ok) continue;
      ok = wait_all(&st.q_full, part & 1u);
      auto issue_s = [&](int j) {
        const int c = p.tiles == 2 ? j >> 1 : j, g = j & 1;
        const uint32_t i = n + items.keys(c), slot = i % SM::kSlots;
        ok = ok && wait_all(&st.slot_full[slot], (i / SM::kSlots) & 1u);
        if (!ok) return;
        tc_fence_after();
        const uint64_t qd = desc_sw128_s(smem_u32(base + SM::kQ + (p.tiles == 2 ? g : 0) * SM::kTile), 16, HD * 16);
        const uint64_t kd = desc_sw128_s(smem_u32(base + SM::kSlot0 + slot * SM::kTile), 16, HD * 16);
        if (elect_lane()) {
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            const uint32_t step = ((k >> 2) * kAtom + (k & 3) * 32) >> 4;
            umma(tmem + kColS + g * 128, qd + step, kd + step, id_s, k > 0 ? 1u : 0u);
          }
        }
        __syncwarp();
        umma_commit_w(&st.s_full[g]);
        if (p.tiles == 1 || g == 1) umma_commit_w(&st.slot_empty[slot]);
        if (j == units - 1) umma_commit_w(&st.q_empty);
      };
      auto issue_o = [&](int j) {
        const int c = p.tiles == 2 ? j >> 1 : j, g = j & 1;
        const uint32_t i = n + items.values(c), slot = i % SM::kSlots;
        ok = ok && wait_all(&st.slot_full[slot], (i / SM::kSlots) & 1u);
        ok = ok && wait_all(&st.p_full[g], (phase >> g) & 1u);
        phase ^= 1u << g;
        if (!ok) return;
        uint8_t* tile = base + SM::kSlot0 + slot * SM::kTile;
        if constexpr (!E4M3) {
          // the last cached chunk's last page: its places beyond the length may hold anything, and a weight of
          // zero would keep a NaN
          const int have = p.q.len - (p.c0 + c) * kChunk;
          if (p.c0 + c == p.q.cached_blocks - 1 && (have & 15) != 0 && (p.tiles == 1 || g == 0)) {
            const int rows = 16 - (have & 15);
            for (int x = lane; x < rows * (HD / 8); x += 32)
              *reinterpret_cast<uint4*>(tile + swizzled<HD>(have + x / (HD / 8), x % (HD / 8))) =
                  make_uint4(0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
            __syncwarp();
          }
        }
        tc_fence_after();
        const uint64_t vd = desc_sw128_s(smem_u32(tile), kAtom, HD * 16);
        const uint32_t pt = tmem + kColS + g * 128;
        if (elect_lane()) {
#pragma unroll
          for (int k = 0; k < kChunk / 16; ++k)
            umma_ta(tmem + kColO + g * 128, pt + k * 8, vd + (k * (HD * 32) >> 4), id_o, k > 0 || j >= 2 ? 1u : 0u);
        }
        __syncwarp();
        if (p.tiles == 1 || g == 1) umma_commit_w(&st.slot_empty[slot]);
      };
      if (ok) issue_s(0);
      if (units > 1) issue_s(1);
      if (part > 0) ok = ok && wait_all(&st.o_free, (part - 1) & 1u);   // the accumulators are read out
      for (int j = 0; j < units && ok; ++j) {
        issue_o(j);
        if (j + 2 < units && ok) issue_s(j + 2);
      }
      if (ok) umma_commit_w(&st.part_done);
      n += items.n;
    }
  } else if (warp >= 8 && warp < 16) {
    // ------------------------------------------------ producers
    const int t = threadIdx.x - 256;
    uint32_t n = 0, go = 0;   // go: per slot, the parity of its next draft_go
    bool ok = true;
    auto filled = [&](uint64_t* bar) {   // this tile's writes, seen by the tensor cores, then its barrier
      fence_proxy_async_smem();
      named_bar_sync(2, kProducers);
      if (t == 0) mbar_arrive(bar);
    };
    auto slot_filled = [&](uint64_t* bar) {   // a slot's: with an 8-bit cache each warp goes on by itself
      if constexpr (E4M3) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      } else {
        filled(bar);
      }
    };
    // An 8-bit chunk's keys or values: a warp has one page, whose codes it loads an item ahead and converts kTeam rows at
    // a time; it waits for slots and hands them on by itself.  A row's 8 pieces fill two 64-column parts, whose equal
    // pieces lie in the same banks: lanes 0 to 3 and 4 to 7 take neighbouring rows, which the swizzle puts in different
    // ones.
    constexpr int kParts = HD / 16, kTeam = 32 / kParts, kSteps = kTreePage / kTeam;   // 16-byte pieces of a row
    const int my_page = t >> 5, my_piece = lane % kParts;
    const int my_row = HD == 128 ? (lane >> 4) * 2 + (((lane >> 3) & 1) ^ (my_piece >> 2)) : lane / kParts;   // of a step's
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;   // a negative scale turns Q's signs instead
    for (int part = 0; next_part(); ++part) {
      const int rows = p.q.drafts * a.group;
      const Items items(p);
      const int32_t* table = a.t.block_table + static_cast<int64_t>(a.seq0 + p.s) * a.t.max_blocks;
      const int pages = (p.q.len + kTreePage - 1) / kTreePage;
      auto page_of = [&](int item) {   // -1: no page there, -2: not a page of the cache
        int kv;
        const int at = item < items.n ? (p.c0 + items.chunk(item, &kv)) * kPages + my_page : pages;
        if (at >= pages) return -1;
        const int32_t page = __ldg(table + at);
        return page < 0 || page >= a.n_pages ? -2 : page;
      };
      uint32_t bad = 0;   // items (modulo 4) with a page outside the cache
      uint4 next[kSteps];
      uint32_t next_e = 0;
      auto load = [&](int item, int32_t page) {
        if (page == -2) bad |= 1u << (item & 3);
        if (page < 0) return;
        int kv;
        items.chunk(item, &kv);
        const int64_t row = ((static_cast<int64_t>(page) * 2 + kv) * a.n_kv + p.g) * kTreePage;
        const uint8_t* src = a.pages + row * HD + my_row * HD + my_piece * 16;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) next[k] = ldg_stream(src + k * 512);
        next_e = __ldg(a.exponents + row + lane % kTreePage);
      };
      int32_t page = -1;
      if constexpr (E4M3) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) next[k] = make_uint4(0u, 0u, 0u, 0u);
        const int32_t page0 = page_of(0);
        page = page_of(1);
        load(0, page0);
      }
      if (part > 0) ok = ok && wait_for(&st.q_empty, (part - 1) & 1u, err);
      constexpr int kPieces = HD / 8, kStep = kProducers / kPieces;   // a thread's rows are kStep apart
      for (int tile = 0; tile < p.tiles; ++tile) {
        uint8_t* dst = base + SM::kQ + tile * SM::kTile;
        const int piece = t % kPieces, first = t / kPieces, left = rows - (2 * p.tp + tile) * kRows;
        uint4 v[kRows / kStep];   // all loads in flight
#pragma unroll
        for (int i = 0; i < kRows / kStep; ++i) {
          const int r = first + i * kStep;
          v[i] = make_uint4(0u, 0u, 0u, 0u);
          if (r < left) {
            const int row = rows - left + r, tok = tree_token(a, row), h = p.g * a.group + row - tok * a.group;
            v[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.t.q) +
                                                        (p.q.start + static_cast<int64_t>(tok)) * a.t.q_token +
                                                        h * a.t.q_head) + piece);
          }
        }
#pragma unroll
        for (int i = 0; i < kRows / kStep; ++i) {
          v[i] = make_uint4(v[i].x ^ flip, v[i].y ^ flip, v[i].z ^ flip, v[i].w ^ flip);
          *reinterpret_cast<uint4*>(dst + swizzled<HD>(first + i * kStep, piece)) = E4M3 ? paired(v[i]) : v[i];
        }
      }
      filled(&st.q_full);
      for (int item = 0; item < items.n; ++item) {
        int kv;
        const int c = p.c0 + items.chunk(item, &kv);
        const bool cached = c < p.q.cached_blocks;
        if (cached && !E4M3) continue;
        const uint32_t i = n + item, slot = i % SM::kSlots;
        uint8_t* dst = base + SM::kSlot0 + slot * SM::kTile;
        if constexpr (E4M3) {   // every slot is filled here
          if (i >= SM::kSlots) ok = ok && wait_for(&st.slot_empty[slot], (i / SM::kSlots - 1) & 1u, err);
          uint4 codes[kSteps];
#pragma unroll
          for (int k = 0; k < kSteps; ++k) codes[k] = next[k];
          const uint32_t e = next_e;
          load(item + 1, page);
          page = page_of(item + 2);
          if (cached) {
            if (lane == 0 && (bad >> (item & 3)) & 1u) atomicOr(&st.bad[part % kFlagSets], 1);
            bad &= ~(1u << (item & 3));
            // the factor of a row, per lane: 2^(e - 127 + 120) as bf16, beyond its range (or NaN, 255) in two; zero past the
            // length, where the codes may be anything
            const bool live = my_page * kTreePage + lane % kTreePage < p.q.len - c * kChunk, two = e > 134u && live;
            uint32_t f = (two ? 254u : e + 120u) << 7 | (two ? (e == 255u ? 0x7FC0u : (e - 7u) << 7) : 0x3F80u) << 16;
            if (!live) f = 0x3F800000u;
            // (126 rows of 4 heads over 16 x 9,001 tokens: 84 us without the check for NaN codes, 86 with it, 91 with a vote and a
            // loop of its own, whose loads made every item wait for those ahead)
            uint32_t carries = 0;
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
              carries |= nan_carries(codes[k].x) | nan_carries(codes[k].y) | nan_carries(codes[k].z) | nan_carries(codes[k].w);
            auto convert = [&](auto plain) {
#pragma unroll
              for (int k = 0; k < kSteps; ++k) {
                const uint32_t fr = __shfl_sync(0xffffffffu, f, my_row + kTeam * k);
                uint4 lo, hi;
                bf16_of16<decltype(plain)::value>(codes[k], __byte_perm(fr, 0, 0x1010), __byte_perm(fr, 0, 0x3232), &lo, &hi);
                const int row = my_page * kTreePage + k * kTeam + my_row;
                *reinterpret_cast<uint4*>(dst + swizzled<HD>(row, 2 * my_piece)) = lo;
                *reinterpret_cast<uint4*>(dst + swizzled<HD>(row, 2 * my_piece + 1)) = hi;
              }
            };
            if (__any_sync(0xffffffffu, two || (carries & 0x80808080u) != 0u))
              convert(std::false_type());
            else
              convert(std::true_type());
            slot_filled(&st.slot_full[slot]);
            continue;
          }
        } else {
          ok = ok && wait_for(&st.draft_go[slot], (go >> slot) & 1u, err);
          go ^= 1u << slot;
        }
        // ---- drafted tokens: bf16 rows of their own tensors, whatever the cache holds
        const int j0 = (c - p.q.cached_blocks) * kChunk, have = p.q.drafts - j0;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(kv ? a.t.v : a.t.k) +
                                   (p.q.start + static_cast<int64_t>(j0)) * (kv ? a.t.v_token : a.t.k_token) +
                                   p.g * (kv ? a.t.v_head : a.t.k_head);
        const int64_t step = kv ? a.t.v_token : a.t.k_token;
#pragma unroll 2
        for (int x = t; x < kChunk * kPieces; x += kProducers) {   // a row's pieces: neighbouring lanes of a warp
          const int row = x / kPieces, piece = x % kPieces;
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (row < have) v = __ldg(reinterpret_cast<const uint4*>(src + row * step) + piece);
          if (kv) {   // a weight of zero must leave no trace of a value that is not finite: its readers are marked
            const bool off = not_finite2(v.x) || not_finite2(v.y) || not_finite2(v.z) || not_finite2(v.w);
            const uint32_t who = __ballot_sync(0xffffffffu, off);
            if ((who >> (lane / kPieces * kPieces)) & ((1u << kPieces) - 1u)) {
              v = make_uint4(0u, 0u, 0u, 0u);
              if (piece == 0) {
                atomicOr(&st.bad_drafts[part % kFlagSets][(j0 + row) >> 5], 1u << ((j0 + row) & 31));
                atomicOr(&st.bad[part % kFlagSets], 2);
              }
            }
          }
          *reinterpret_cast<uint4*>(dst + swizzled<HD>(row, piece)) = E4M3 ? paired(v) : v;
        }
        slot_filled(&st.slot_full[slot]);
      }
      n += items.n;
    }
  } else if (warp < 8) {
    // ------------------------------------------------ softmax
    const int g = warp >> 2, r = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + kColS + g * 128, to = tmem + lanes + kColO;
    const float scale = fabsf(a.scale_log2);
    float2* s_ml = reinterpret_cast<float2*>(base + SM::kMl);
    uint32_t uses = 0;
    bool ok = true;
    for (int part = 0; next_part(); ++part) {
      TreePart& sp = st.part[warp];
      __syncwarp();
      if (lane == 0) {
        sp = p;
        st.walk[warp] = make_int4(u, u_end, s, 0);
      }
      __syncwarp();
      const bool both = sp.tiles == 2;   // the groups have a tile each, else alternate chunks of one
      const int rows = sp.q.drafts * a.group, row = (2 * sp.tp + (both ? g : 0)) * kRows + r;
      const bool live = row < rows, warp_live = row - lane < rows;   // (a dead row's weights, whatever they are, stay in it)
      const int tok = live ? tree_token(a, row) : 0;
      float m = -INFINITY, l = 0.f;
      bool begun = false;
      for (int c = both ? sp.c0 : sp.c0 + g; c < sp.c1; c += both ? 1 : 2) {
        const bool cached = c < sp.q.cached_blocks;
        // which of the chunk's keys this row sees
        uint32_t sees[4] = {~0u, ~0u, ~0u, ~0u};
        bool all = true;
        if (cached) {
          const int have = sp.q.len - c * kChunk;
          if (have < kChunk) {
            all = false;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int left = have - 32 * w;
              sees[w] = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1u;
            }
          }
        } else {
          all = false;
          const int j0 = (c - sp.q.cached_blocks) * kChunk;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int j = j0 + 32 * w;
            sees[w] = live && j < sp.q.drafts
                          ? tree_sees16(a, sp.q, tok, j) | (j + 16 < sp.q.drafts ? tree_sees16(a, sp.q, tok, j + 16) << 16 : 0u)
                          : 0u;
          }
        }
        ok = ok && __all_sync(0xffffffffu, wait_for(&st.s_full[g], uses & 1u, err));
        tc_fence_after();
        if (ok && warp_live) {
          // Two passes over the row's S, 16 columns at a time with the next ones on their way: its maximum, then the
          // weights.  (SEEN: every key; the other form is for a cache's last chunk and for drafted tokens.)
          float x[2][16];
          auto arrived = [&](int b) {
            tmem_wait_ld();
            tmem_hold(x[b]);
          };
          auto bits_of = [&](int h) {   // of the keys of columns 16 h ..
            const uint32_t w = h < 4 ? (h < 2 ? sees[0] : sees[1]) : (h < 6 ? sees[2] : sees[3]);
            return w >> (16 * (h & 1));
          };
          float mx = -INFINITY;
          tmem_ld16_nowait(ts, x[0]);
          if (all) {
            float my = -INFINITY;
#pragma unroll
            for (int h = 0; h < 8; ++h) {
              arrived(h & 1);
              tmem_ld16_nowait(ts + (h < 7 ? (h + 1) * 16 : 0), x[(h + 1) & 1]);   // (at the end the first ones again, for the weights)
              const float(&y)[16] = x[h & 1];
#pragma unroll
              for (int i = 0; i < 16; i += 4) {
                mx = fmaxf(mx, fmaxf(y[i], y[i + 1]));
                my = fmaxf(my, fmaxf(y[i + 2], y[i + 3]));
              }
            }
            mx = fmaxf(mx, my);
          } else {
#pragma unroll 1
            for (int h = 0; h < 8; ++h) {
              tmem_ld16(ts + h * 16, x[0]);   // (waits)
              const uint32_t bits = bits_of(h);
#pragma unroll
              for (int i = 0; i < 16; ++i) mx = fmaxf(mx, (bits >> i) & 1u ? x[0][i] : -INFINITY);
            }
          }
          mx *= scale;
          if (scale == 0.f && mx != mx) mx = 0.f;   // -infinity times zero: nothing seen, or scores of zero
          const bool grow = mx > m + kMargin;
          if (__any_sync(0xffffffffu, grow) && begun) {   // the accumulator follows (every MMA on it has completed)
            const float f = grow ? (m == -INFINITY ? 0.f : ex2_ftz(m - mx)) : 1.f;
#pragma unroll 1
            for (int i = 0; i < HD; i += 16) {
              float o[16];
              tmem_ld16(to + g * 128 + i, o);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] *= f;
              tmem_st16(to + g * 128 + i, o);
            }
            tmem_wait_st();
          }
          if (grow) {
            l = m == -INFINITY ? l : l * ex2_ftz(m - mx);
            m = mx;
          }
          begun = true;
          const float nm = m == -INFINITY ? 0.f : -m;
          float2 sum = make_float2(0.f, 0.f), sum1 = sum;
          const float2 scale2 = make_float2(scale, scale), nm2 = make_float2(nm, nm);
          // the weights go as bf16 (the values' type) over columns of S that have been read
          if (all) {
#pragma unroll
            for (int h = 0; h < 8; ++h) {
              arrived(h & 1);
              if (h < 7) tmem_ld16_nowait(ts + (h + 1) * 16, x[(h + 1) & 1]);
              float w[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float2 y = fma2(make_float2(x[h & 1][2 * i], x[h & 1][2 * i + 1]), scale2, nm2);
                y = make_float2(ex2_ftz(y.x), ex2_ftz(y.y));
                (i & 1 ? sum1 : sum) = add2(i & 1 ? sum1 : sum, y);
                w[i] = __uint_as_float(pack_bf16(y.x, y.y));
              }
              tmem_st8(ts + h * 8, w);
            }
          } else {
#pragma unroll 1
            for (int h = 0; h < 8; ++h) {
              tmem_ld16(ts + h * 16, x[0]);
              const uint32_t bits = bits_of(h);
              float w[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float2 y = fma2(make_float2(x[0][2 * i], x[0][2 * i + 1]), scale2, nm2);
                y = make_float2((bits >> (2 * i)) & 1u ? ex2_ftz(y.x) : 0.f, (bits >> (2 * i + 1)) & 1u ? ex2_ftz(y.y) : 0.f);
                sum = add2(sum, y);
                w[i] = __uint_as_float(pack_bf16(y.x, y.y));
              }
              tmem_st8(ts + h * 8, w);
            }
          }
          l += (sum.x + sum1.x) + (sum.y + sum1.y);
          tmem_wait_st();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&st.p_full[g]);
        ++uses;
      }

      // ---- the part's end
      ok = ok && __all_sync(0xffffffffu, wait_for(&st.part_done, part & 1u, err));
      tc_fence_after();
      const int set = part % kFlagSets, marks = st.bad[set];
      bool nan = !ok || sp.q.bad || (marks & 1) != 0;
      if ((marks & 2) && live) {
        for (int j = 0; j < sp.q.drafts; j += 16)
          if (tree_sees16(a, sp.q, tok, j) & (st.bad_drafts[set][j >> 5] >> (j & 31))) nan = true;
      }
      if (nan) l = NAN;
      s_ml[g * kRows + r] = make_float2(m, l);
      named_bar_sync(1, 256);
      // one tile: both groups' states of the row, and each group half of its dimensions; two: all of its own row
      const float2 mine = s_ml[(both ? g : 0) * kRows + r], other = both ? make_float2(-INFINITY, 0.f) : s_ml[kRows + r];
      if (threadIdx.x < 32) {   // (the marks have been read) clean for a later part
        st.bad_drafts[set][threadIdx.x] = 0;
        if (threadIdx.x == 0) st.bad[set] = 0;
      }
      const float top = fmaxf(mine.x, other.x);
      auto factor = [](float2 ml, float best) { return ml.x == -INFINITY ? 0.f : ex2_ftz(ml.x - best); };   // (NaN sums stay NaN)
      const float f0 = factor(mine, top), f1 = factor(other, top);
      const float sum = mine.y * f0 + other.y * f1;
      const bool two_streams = !both && sp.c1 - sp.c0 > 1;   // else the second accumulator holds nothing of this part
      const int d_begin = both ? 0 : g * (HD / 2), d_end = both ? HD : d_begin + HD / 2;
      const bool whole = sp.whole();
      // a partial result: [dim][row], so that a warp's rows are stored side by side
      const int64_t slot = me == TreeShares(st.off[a.n_seqs], gridDim.x, a.weight_full).owner(sp.place(0)) ? 2 * me + 1 : 2 * me;
      const int slot_row = (both ? g : 0) * kRows + r;
      float* part_o = a.part_o + slot * (HD * TreeTc::kSlotRows) + slot_row;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that saw nothing: zeros
      __nv_bfloat16* dst = nullptr;
      if (live)
        dst = static_cast<__nv_bfloat16*>(a.t.out) + (sp.q.start + static_cast<int64_t>(tok)) * a.t.out_token +
              (sp.g * a.group + row - tok * a.group) * a.t.out_head;
#pragma unroll 1
      for (int d = d_begin; d < d_end; d += 16) {
        float o[16], o1[16];
        __syncwarp();
        if (ok) {
          tmem_ld16_nowait(to + (both ? g : 0) * 128 + d, o);
          if (two_streams) tmem_ld16_nowait(to + 128 + d, o1);
          tmem_wait_ld();
          tmem_hold(o);
          if (two_streams) tmem_hold(o1);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] = ok ? o[i] * f0 + (two_streams ? o1[i] * f1 : 0.f) : 0.f;
        if (E4M3) in_order(o);
        if (!live) continue;
        if (whole) {
          uint32_t w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = pack_bf16(o[2 * i] * inv, o[2 * i + 1] * inv);
          *reinterpret_cast<uint4*>(dst + d) = make_uint4(w[0], w[1], w[2], w[3]);
          *reinterpret_cast<uint4*>(dst + d + 8) = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) part_o[(d + i) * TreeTc::kSlotRows] = o[i];
        }
      }
      if (!whole && live && d_begin == 0) a.part_ml[slot * TreeTc::kSlotRows + slot_row] = make_float2(top, sum);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&st.o_free);
      named_bar_sync(1, 256);   // the states are read before the next part's are written
      u = st.walk[warp].x;
      u_end = st.walk[warp].y;
      s = st.walk[warp].z;
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kWarpMma) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <int HD, bool E4M3>
cudaError_t launch(const TreeLaunch& a, const CUtensorMap& map, int ctas, cudaStream_t stream) {
  using SM = Smem<HD, E4M3>;
  static_assert(SM::kDynamic + sizeof(Static) <= 227 * 1024, "shared memory of a CTA");
  cudaError_t e = cudaFuncSetAttribute(tree_tc_kernel<HD, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(SM::kDynamic));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = SM::kDynamic;
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, tree_tc_kernel<HD, E4M3>, a, map);
}

// Pages [n_pages][2][n_kv][16][hd] as (column of 64, row of 8, 64-column part, half of the page's rows, (2 page + {0: keys,
// 1: values}) n_kv + kv head); a box is one page's keys or values of one head.
CUresult encode_pages(PFN_cuTensorMapEncodeTiled_v12000 encode, CUtensorMap* map, const kvprm_cache& c) {
  const cuuint64_t row = static_cast<cuuint64_t>(c.head_dim) * 2, parts = c.head_dim / 64;
  if (c.n_pages > 0x7FFFFFFF / (2 * int64_t{c.n_kv_heads})) return CUDA_ERROR_INVALID_VALUE;   // coordinates are 32-bit
  const cuuint64_t dims[5] = {64, 8, parts, 2, static_cast<cuuint64_t>(c.n_pages) * 2 * c.n_kv_heads};
  const cuuint64_t strides[4] = {row, 128, 8 * row, kTreePage * row};
  const cuuint32_t box[5] = {64, 8, static_cast<cuuint32_t>(parts), 2, 1}, step[5] = {1, 1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, c.pages, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

}  // namespace

cudaError_t launch_tree_tc(const TreeLaunch& a, const kvprm_cache& c, int ctas, cudaStream_t stream) {
  CUtensorMap map = {};
  if (c.format == KVPRM_CACHE_E4M3)
    return c.head_dim == 128 ? launch<128, true>(a, map, ctas, stream) : launch<64, true>(a, map, ctas, stream);
  static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      fn = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  }();
  if (!encode) return cudaErrorNotSupported;
  if (encode_pages(encode, &map, c) != CUDA_SUCCESS) return cudaErrorInvalidValue;
  return c.head_dim == 128 ? launch<128, false>(a, map, ctas, stream) : launch<64, false>(a, map, ctas, stream);
}

}  // namespace kvprm
