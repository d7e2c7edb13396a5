// Attention of drafted tokens over the paged cache on the tensor cores (tcgen05), for more than 16 query
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
//   warps 8-11       producers: Q tiles, drafted tokens' keys and values, and with an 8-bit cache every chunk,
//                    converted to bf16 (exact: a power of two per row changes no mantissa)
//   warp 12          TMA: bf16 pages straight into the tiles, 8-bit pages into a ring of their own
//   warp 13          issues every MMA, in an order that keeps one unit's S ahead of the other's O
// Tiles lie in shared memory as rows of 128 bytes under the 128-byte swizzle, [64-column part][128 rows]: a
// K-major operand for the keys and an MN-major one for the values.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kernels.h"
#include "ptx.cuh"
#include "rope.h"
#include "tree.h"

namespace kvprm {

namespace {

constexpr int kThreads = 448;
constexpr int kRows = 128, kChunk = 128, kPages = kChunk / kTreePage;
constexpr int kProducers = 128;
constexpr float kMargin = 8.f;   // log2 units that scores may pass a running maximum by
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;   // S buffers at 0 and 128, accumulators at 256 and 384
constexpr int kFlagSets = 4;     // parts whose marks may be in flight (the rings hold chunks of at most three)

template <int HD, bool E4M3>
struct Smem {
  static constexpr uint32_t kTile = kChunk * HD * 2;             // one chunk's keys or values, or one tile of Q
  static constexpr int kSlots = HD == 128 ? (E4M3 ? 3 : 4) : (E4M3 ? 4 : 8);
  static constexpr int kRaw = E4M3 ? (HD == 128 ? 3 : 6) : 1;
  static constexpr uint32_t kRawCodes = kChunk * HD;
  static constexpr uint32_t kRawBytes = kRawCodes + kChunk;      // codes, then the rows' exponents
  static constexpr uint32_t kQ = 0;                              // two tiles
  static constexpr uint32_t kSlot0 = kQ + 2 * kTile;
  static constexpr uint32_t kRaw0 = kSlot0 + kSlots * kTile;
  static constexpr uint32_t kMl = kRaw0 + (E4M3 ? kRaw * kRawBytes : 0);   // float2 [2][128]
  static constexpr uint32_t kEnd = kMl + 2 * kRows * 8;
  static constexpr size_t kDynamic = kEnd + 1024;
};

struct Static {   // in static shared memory
  int64_t off[kTreeSeqs + 1];
  int64_t sum[kThreads / 32];
  uint64_t slot_full[8], slot_empty[8], raw_full[8], raw_empty[8];
  uint64_t draft_go[8];   // bf16 cache: a free slot that is the producers' to fill
  uint64_t q_full, q_empty, s_full[2], p_full[2], part_done, o_free;
  uint32_t bad_drafts[kFlagSets][32];   // drafted tokens of a part whose values are not finite
  int bad[kFlagSets];                   // of a part: a page outside the cache, a bad draft (1, 2)
  int raw_bad[8];                       // a page outside the cache, of a raw slot
  uint32_t tmem;
  int last;
};

// One CTA's part of a pair.
struct Part {
  TreeSeq q;
  int64_t pair0;          // the pair's first place on the line
  int s, g, tp, tiles;    // tiles: 1 or 2, and a chunk's weight on the line
  int c0, c1;             // chunks
};

__device__ __forceinline__ bool next_part(const TreeLaunch& a, const int64_t* off, int64_t& u, int64_t u_end, int& s,
                                          Part& p) {
  while (u < u_end) {
    while (u >= off[s + 1]) ++s;
    p.q = tree_seq<kRows, kChunk>(a, s);
    p.s = s;
    const int64_t head_len = static_cast<int64_t>(p.q.blocks) * p.q.tiles, local = u - off[s];
    p.g = static_cast<int>(local / head_len);
    const int64_t in_head = local - p.g * head_len;
    p.tp = static_cast<int>(in_head / (2 * p.q.blocks));
    p.pair0 = off[s] + p.g * head_len + static_cast<int64_t>(p.tp) * 2 * p.q.blocks;
    p.tiles = min(2, p.q.tiles - 2 * p.tp);
    p.c0 = static_cast<int>((u - p.pair0 + p.tiles - 1) / p.tiles);
    p.c1 = static_cast<int>(min(static_cast<int64_t>(p.q.blocks), (u_end - p.pair0 + p.tiles - 1) / p.tiles));
    u = p.c1 == p.q.blocks ? p.pair0 + static_cast<int64_t>(p.q.blocks) * p.tiles : u_end;
    if (p.c0 < p.c1) return true;
  }
  return false;
}

__device__ __forceinline__ uint32_t swizzled(int row, int piece) {   // of a 16-byte piece of a tile's row
  return static_cast<uint32_t>(piece >> 3) * (kRows * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// Four e4m3 codes as bf16 times a row's power of two.  A code's exponent and mantissa at bf16's place are
// 2^-120 of its value; f1 * f2 is 2^120 times the row's power (f2 = 1 unless that passes bf16's range).
__device__ __forceinline__ uint2 bf16_of4(uint32_t w, uint32_t f1, uint32_t f2, bool two) {
  uint32_t e = ((w << 4) & 0x07F007F0u) | ((w << 8) & 0x80008000u);   // bytes 0, 2
  uint32_t o = ((w >> 4) & 0x07F007F0u) | (w & 0x80008000u);          // bytes 1, 3
  e = mul_bf16x2(e, f1);
  o = mul_bf16x2(o, f1);
  if (two) {
    e = mul_bf16x2(e, f2);
    o = mul_bf16x2(o, f2);
  }
  return make_uint2(__byte_perm(e, o, 0x5410), __byte_perm(e, o, 0x7632));
}

template <int HD, bool E4M3>
__global__ void __launch_bounds__(kThreads, 1) tree_tc_kernel(const __grid_constant__ TreeLaunch a,
                                                              const __grid_constant__ CUtensorMap map) {
  using SM = Smem<HD, E4M3>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Static st;
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t{1023});
  int* err = a.tickets + kTreeTickets - 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 8; ++i) {
      mbar_init(&st.slot_full[i], 1);
      mbar_init(&st.slot_empty[i], 1);
      mbar_init(&st.draft_go[i], 1);
      mbar_init(&st.raw_full[i], 1);
      mbar_init(&st.raw_empty[i], 1);
    }
    mbar_init(&st.q_full, 1);
    mbar_init(&st.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&st.s_full[i], 1);
      mbar_init(&st.p_full[i], 4);
    }
    mbar_init(&st.part_done, 1);
    mbar_init(&st.o_free, 8);
    fence_mbar_init();
    if constexpr (!E4M3) tma_prefetch_desc(&map);
  }
  if (threadIdx.x < kFlagSets * 32) st.bad_drafts[threadIdx.x >> 5][lane] = 0;
  if (threadIdx.x < kFlagSets) st.bad[threadIdx.x] = 0;
  if (warp == 13) {
    tmem_alloc(&st.tmem, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  tree_line<kRows, kChunk, kThreads>(a, st.off, st.sum);   // barriers inside
  tc_fence_after();
  const uint32_t tmem = st.tmem;
  const int64_t total = st.off[a.n_seqs];
  // a share of two or more holds at least one chunk's start of any pair that it lies in
  const int P = static_cast<int>(min(static_cast<int64_t>(gridDim.x), max(total / 2, int64_t{1})));
  const int me = blockIdx.x;
  const bool idle = me >= P || total == 0;
  int64_t u = idle ? 0 : total * me / P;
  const int64_t u_end = idle ? 0 : total * (me + 1) / P;
  int s = idle ? 0 : tree_find(st.off, a.n_seqs, u);
  Part p;

  if (warp == 12) {
    // ------------------------------------------------ TMA
    const uint64_t pol = policy_evict_normal();
    uint32_t n = 0;   // items: keys of chunk 0, values of chunk 0, keys of chunk 1 ...
    uint32_t loaded = 0;
    bool ok = true;
    auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, err)); };
    for (int part = 0; ok && next_part(a, st.off, u, u_end, s, p); ++part) {
      const int32_t* table = a.t.block_table + static_cast<int64_t>(a.seq0 + p.s) * a.t.max_blocks;
      const int pages = (p.q.len + kTreePage - 1) / kTreePage;
      for (int c = p.c0; c < p.c1 && ok; ++c, n += 2) {
        const bool cached = c < p.q.cached_blocks;
        if (E4M3 && !cached) continue;
        // lane i < 8: the chunk's i-th page (-1: none there, -2: not a page of the cache)
        const int at = c * kPages + lane;
        int32_t page = -1;
        if (cached && lane < kPages && at < pages) {
          page = __ldg(table + at);
          if (page < 0 || page >= a.n_pages) page = -2;
        }
        const bool bad = __any_sync(0xffffffffu, page == -2);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if constexpr (E4M3) {
            const uint32_t r = loaded % SM::kRaw;
            if (loaded >= SM::kRaw) ok = ok && wait_all(&st.raw_empty[r], (loaded / SM::kRaw - 1) & 1u);
            if (!ok) break;
            constexpr uint32_t kPageBytes = kTreePage * HD;
            const uint32_t good = __popc(__ballot_sync(0xffffffffu, page >= 0));
            if (lane == 0) {
              st.raw_bad[r] = bad;
              mbar_arrive_expect_tx(&st.raw_full[r], good * (kPageBytes + kTreePage));
            }
            __syncwarp();
            if (page >= 0) {
              uint8_t* dst = base + SM::kRaw0 + r * SM::kRawBytes;
              const int64_t row = (static_cast<int64_t>(page) * 2 + kv) * a.n_kv + p.g;
              bulk_load(dst + lane * kPageBytes, a.pages + row * kPageBytes, kPageBytes, &st.raw_full[r]);
              bulk_load(dst + SM::kRawCodes + lane * kTreePage, a.exponents + row * kTreePage, kTreePage, &st.raw_full[r]);
            }
            __syncwarp();
            ++loaded;
          } else {
            // This warp waits for every use of a slot, also where the producers fill it: a wait by parity sees only
            // the phase before the present one, so none may be left out.
            const uint32_t i = n + kv, slot = i % SM::kSlots;
            if (i >= SM::kSlots) ok = ok && wait_all(&st.slot_empty[slot], (i / SM::kSlots - 1) & 1u);
            if (!ok) break;
            if (!cached) {
              if (lane == 0) mbar_arrive(&st.draft_go[slot]);
              continue;
            }
            if (lane == 0) {
              // (a part's marks are set once a slot of it is free: no earlier part then holds the same set)
              if (bad) atomicOr(&st.bad[part % kFlagSets], 1);
              mbar_arrive_expect_tx(&st.slot_full[slot], SM::kTile);
            }
            __syncwarp();
            // lane (sub, page): a 2 KB box of 16 rows of 64 columns; places without a page read one that does
            // not exist and arrive as zeros
            const int32_t pg = __shfl_sync(0xffffffffu, page, lane % kPages);
            const int sub = lane / kPages;
            if (sub < HD / 64)
              tma_load_5d(base + SM::kSlot0 + slot * SM::kTile + sub * (kRows * 128) + (lane % kPages) * 2048, &map,
                          &st.slot_full[slot], 0, 0, sub, p.g, pg >= 0 ? 2 * pg + kv : -1, pol);
            __syncwarp();
          }
        }
      }
    }
    // Nothing of this warp's is in flight when the CTA ends: the matrix products (or the producers) waited for every
    // load.  After a wait that gave up, a millisecond is far beyond a load's time.
    if (!ok) {
      const uint64_t t0 = global_timer_ns();
      while (global_timer_ns() - t0 < 1000000ull) __nanosleep(1000);
    }
  } else if (warp == 13) {
    // ------------------------------------------------ MMA
    const uint32_t id_s = idesc_bf16_f32(kRows, kChunk), id_o = idesc_bf16_f32(kRows, HD) | kIdescMnMajorB;
    auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, err)); };
    uint32_t n = 0, uses[2] = {0, 0};
    bool ok = true;
    for (int part = 0; next_part(a, st.off, u, u_end, s, p); ++part) {
      const int chunks = p.c1 - p.c0, units = chunks * p.tiles;
      if (!ok) continue;
      ok = wait_all(&st.q_full, part & 1u);
      auto issue_s = [&](int j) {
        const int c = p.tiles == 2 ? j >> 1 : j, g = j & 1;
        const uint32_t i = n + 2 * c, slot = i % SM::kSlots;
        ok = ok && wait_all(&st.slot_full[slot], (i / SM::kSlots) & 1u);
        if (!ok) return;
        tc_fence_after();
        const uint64_t qd = desc_sw128(smem_u32(base + SM::kQ + (p.tiles == 2 ? g : 0) * SM::kTile));
        const uint64_t kd = desc_sw128(smem_u32(base + SM::kSlot0 + slot * SM::kTile));
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint32_t step = ((k >> 2) * (kRows * 128) + (k & 3) * 32) >> 4;
          umma_bf16_w(tmem + kColS + g * 128, qd + step, kd + step, id_s, k > 0 ? 1u : 0u);
        }
        umma_commit_w(&st.s_full[g]);
        if (p.tiles == 1 || g == 1) umma_commit_w(&st.slot_empty[slot]);
        if (j == units - 1) umma_commit_w(&st.q_empty);
      };
      auto issue_o = [&](int j) {
        const int c = p.tiles == 2 ? j >> 1 : j, g = j & 1;
        const uint32_t i = n + 2 * c + 1, slot = i % SM::kSlots;
        ok = ok && wait_all(&st.slot_full[slot], (i / SM::kSlots) & 1u);
        ok = ok && wait_all(&st.p_full[g], uses[g]++ & 1u);
        if (!ok) return;
        uint8_t* tile = base + SM::kSlot0 + slot * SM::kTile;
        if constexpr (!E4M3) {
          // the last cached chunk's last page: its places beyond the length may hold anything, and a weight of
          // zero would keep a NaN
          const int have = p.q.len - (p.c0 + c) * kChunk;
          if (p.c0 + c == p.q.cached_blocks - 1 && (have & 15) != 0 && (p.tiles == 1 || g == 0)) {
            const int rows = 16 - (have & 15);
            for (int x = lane; x < rows * (HD / 8); x += 32)
              *reinterpret_cast<uint4*>(tile + swizzled(have + x / (HD / 8), x % (HD / 8))) = make_uint4(0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
            __syncwarp();
          }
        }
        tc_fence_after();
        const uint64_t vd = desc_sw128_mn(smem_u32(tile), kRows * 128);
        const uint32_t pt = tmem + kColS + g * 128;
#pragma unroll
        for (int k = 0; k < kChunk / 16; ++k)
          umma_bf16_ta_w(tmem + kColO + g * 128, pt + k * 8, vd + 128 * k, id_o, k > 0 || j >= 2 ? 1u : 0u);
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
      n += 2 * chunks;
    }
  } else if (warp >= 8 && warp < 12) {
    // ------------------------------------------------ producers
    const int t = threadIdx.x - 256;
    uint32_t n = 0, raw = 0, go = 0;   // go: per slot, the parity of its next draft_go
    bool ok = true;
    auto filled = [&](uint64_t* bar) {   // this tile's writes, seen by the tensor cores, then its barrier
      fence_proxy_async_smem();
      named_bar_sync(2, kProducers);
      if (t == 0) mbar_arrive(bar);
    };
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;   // a negative scale turns Q's signs instead
    for (int part = 0; next_part(a, st.off, u, u_end, s, p); ++part) {
      const int rows = p.q.drafts * a.group;
      if (part > 0) ok = ok && mbar_wait(&st.q_empty, (part - 1) & 1u, err);
      constexpr int kPieces = HD / 8;
      for (int tile = 0; tile < p.tiles; ++tile) {
        uint8_t* dst = base + SM::kQ + tile * SM::kTile;
#pragma unroll 4
        for (int x = t; x < kRows * kPieces; x += kProducers) {
          const int r = x / kPieces, piece = x % kPieces, row = (2 * p.tp + tile) * kRows + r;
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (row < rows) {
            const int tok = row / a.group, h = p.g * a.group + row - tok * a.group;
            v = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.t.q) +
                                                     (p.q.start + static_cast<int64_t>(tok)) * a.t.q_token +
                                                     h * a.t.q_head) + piece);
            v = make_uint4(v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip);
          }
          *reinterpret_cast<uint4*>(dst + swizzled(r, piece)) = v;
        }
      }
      filled(&st.q_full);
      for (int c = p.c0; c < p.c1; ++c, n += 2) {
        const bool cached = c < p.q.cached_blocks;
        if (cached && !E4M3) continue;
#pragma unroll 1
        for (int kv = 0; kv < 2; ++kv) {
          const uint32_t i = n + kv, slot = i % SM::kSlots;
          if constexpr (E4M3) {   // every slot is filled here
            if (i >= SM::kSlots) ok = ok && mbar_wait(&st.slot_empty[slot], (i / SM::kSlots - 1) & 1u, err);
          } else {
            ok = ok && mbar_wait(&st.draft_go[slot], (go >> slot) & 1u, err);
            go ^= 1u << slot;
          }
          uint8_t* dst = base + SM::kSlot0 + slot * SM::kTile;
          if (cached) {
            const uint32_t r = raw % SM::kRaw;
            ok = ok && mbar_wait(&st.raw_full[r], (raw / SM::kRaw) & 1u, err);
            if (t == 0 && st.raw_bad[r]) atomicOr(&st.bad[part % kFlagSets], 1);
            const uint8_t* src = base + SM::kRaw0 + r * SM::kRawBytes;
            const int have = min(kChunk, p.q.len - c * kChunk);
            constexpr int kParts = HD / 16;   // 16 codes each
#pragma unroll 4
            for (int x = t; x < kChunk * kParts; x += kProducers) {
              const int row = x / kParts, piece = x % kParts;
              uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
              if (row < have) {
                const uint4 w = *reinterpret_cast<const uint4*>(src + row * HD + piece * 16);
                const uint32_t e = src[SM::kRawCodes + row];
                // 2^(e - 127 + 120) as bf16; beyond its range (or NaN, 255) in two factors
                const bool two = e > 134u;
                const uint32_t f1 = (two ? 254u : e + 120u) << 7, f2 = e == 255u ? 0x7FC0u : (e - 7u) << 7;
                const uint32_t p1 = f1 * 0x10001u, p2 = f2 * 0x10001u;
                const uint2 a0 = bf16_of4(w.x, p1, p2, two), a1 = bf16_of4(w.y, p1, p2, two);
                const uint2 a2 = bf16_of4(w.z, p1, p2, two), a3 = bf16_of4(w.w, p1, p2, two);
                lo = make_uint4(a0.x, a0.y, a1.x, a1.y);
                hi = make_uint4(a2.x, a2.y, a3.x, a3.y);
              }
              *reinterpret_cast<uint4*>(dst + swizzled(row, 2 * piece)) = lo;
              *reinterpret_cast<uint4*>(dst + swizzled(row, 2 * piece + 1)) = hi;
            }
            ++raw;
            filled(&st.slot_full[slot]);
            if (t == 0) mbar_arrive(&st.raw_empty[r]);
          } else {
            const int j0 = (c - p.q.cached_blocks) * kChunk, have = p.q.drafts - j0;
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(kv ? a.t.v : a.t.k) +
                                       (p.q.start + static_cast<int64_t>(j0)) * (kv ? a.t.v_token : a.t.k_token) +
                                       p.g * (kv ? a.t.v_head : a.t.k_head);
            const int64_t step = kv ? a.t.v_token : a.t.k_token;
#pragma unroll 4
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
              *reinterpret_cast<uint4*>(dst + swizzled(row, piece)) = v;
            }
            filled(&st.slot_full[slot]);
          }
        }
      }
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
    for (int part = 0; next_part(a, st.off, u, u_end, s, p); ++part) {
      const bool both = p.tiles == 2;   // the groups have a tile each, else alternate chunks of one
      const int rows = p.q.drafts * a.group, row = (2 * p.tp + (both ? g : 0)) * kRows + r;
      const bool live = row < rows;
      const int tok = live ? row / a.group : 0;
      float m = -INFINITY, l = 0.f;
      bool begun = false;
      for (int c = both ? p.c0 : p.c0 + g; c < p.c1; c += both ? 1 : 2) {
        const bool cached = c < p.q.cached_blocks;
        // which of the chunk's keys this row sees
        uint32_t sees[4] = {~0u, ~0u, ~0u, ~0u};
        bool all = true;
        if (cached) {
          const int have = p.q.len - c * kChunk;
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
          const int j0 = (c - p.q.cached_blocks) * kChunk;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int j = j0 + 32 * w;
            sees[w] = live && j < p.q.drafts
                          ? tree_sees16(a, p.q, tok, j) | (j + 16 < p.q.drafts ? tree_sees16(a, p.q, tok, j + 16) << 16 : 0u)
                          : 0u;
          }
        }
        ok = ok && __all_sync(0xffffffffu, mbar_wait(&st.s_full[g], uses & 1u, err));
        tc_fence_after();
        if (ok) {
          float mx = -INFINITY;
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            float x0[16], x1[16];
            tmem_ld16_nowait(ts + h * 32, x0);
            tmem_ld16_nowait(ts + h * 32 + 16, x1);
            tmem_wait_ld();
            tmem_hold(x0);
            tmem_hold(x1);
            if (all) {
#pragma unroll
              for (int i = 0; i < 16; ++i) mx = fmaxf(mx, fmaxf(x0[i], x1[i]));
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i)
                mx = fmaxf(mx, fmaxf((sees[h] >> i) & 1u ? x0[i] : -INFINITY, (sees[h] >> (16 + i)) & 1u ? x1[i] : -INFINITY));
            }
          }
          mx *= scale;
          if (scale == 0.f && mx != mx) mx = 0.f;   // -infinity times zero: nothing seen, or scores of zero
          const bool grow = mx > m + kMargin;
          const float to_m = grow ? mx : m;
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
            m = to_m;
          }
          begun = true;
          const float nm = m == -INFINITY ? 0.f : -m;
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            float x0[16], x1[16], w[16];
            tmem_ld16_nowait(ts + h * 32, x0);
            tmem_ld16_nowait(ts + h * 32 + 16, x1);
            tmem_wait_ld();
            tmem_hold(x0);
            tmem_hold(x1);
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              x0[i] = ex2_ftz(fmaf(x0[i], scale, nm));
              x1[i] = ex2_ftz(fmaf(x1[i], scale, nm));
              if (!all) {
                x0[i] = (sees[h] >> i) & 1u ? x0[i] : 0.f;
                x1[i] = (sees[h] >> (16 + i)) & 1u ? x1[i] : 0.f;
              }
              l0 += x0[i];
              l1 += x1[i];
            }
            l += l0 + l1;
            // the weights as bf16 (the values' type) over columns of S that have been read
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              w[i] = __uint_as_float(pack_bf16(x0[2 * i], x0[2 * i + 1]));
              w[8 + i] = __uint_as_float(pack_bf16(x1[2 * i], x1[2 * i + 1]));
            }
            tmem_st16(ts + h * 16, w);
          }
          tmem_wait_st();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&st.p_full[g]);
        ++uses;
      }

      // ---- the part's end
      ok = ok && __all_sync(0xffffffffu, mbar_wait(&st.part_done, part & 1u, err));
      tc_fence_after();
      const int set = part % kFlagSets, marks = st.bad[set];
      bool nan = !ok || p.q.bad || (marks & 1) != 0;
      if ((marks & 2) && live) {
        for (int j = 0; j < p.q.drafts; j += 16)
          if (tree_sees16(a, p.q, tok, j) & (st.bad_drafts[set][j >> 5] >> (j & 31))) nan = true;
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
      auto factor = [&](float2 ml, float best) { return ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : ex2_ftz(ml.x - best); };
      const float f0 = factor(mine, top), f1 = factor(other, top);
      float sum = mine.y * f0 + other.y * f1;
      const bool two_streams = !both && p.c1 - p.c0 > 1;   // else the second accumulator holds nothing of this part
      const int d_begin = both ? 0 : g * (HD / 2), d_end = both ? HD : d_begin + HD / 2;
      const bool whole = p.c0 == 0 && p.c1 == p.q.blocks;
      const int slot_row = (both ? g : 0) * kRows + r;
      __nv_bfloat16* dst = nullptr;
      if (live)
        dst = static_cast<__nv_bfloat16*>(a.t.out) + (p.q.start + static_cast<int64_t>(tok)) * a.t.out_token +
              (p.g * a.group + row - tok * a.group) * a.t.out_head;
      auto put = [&](int d, const float (&o)[16], float inv) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack_bf16(o[2 * i] * inv, o[2 * i + 1] * inv);
        *reinterpret_cast<uint4*>(dst + d) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(dst + d + 8) = make_uint4(w[4], w[5], w[6], w[7]);
      };
      int i0 = me, i1 = me;
      if (!whole) {
        i0 = tree_owner(p.pair0, total, P);
        i1 = tree_owner(p.pair0 + static_cast<int64_t>(p.q.blocks - 1) * p.tiles, total, P);
      }
      const int64_t mine_at = static_cast<int64_t>(me == i0 ? 2 * me + 1 : 2 * me) * (2 * kRows) + slot_row;
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
        if (whole) {
          if (live) put(d, o, sum == 0.f ? 0.f : 1.f / sum);   // a row that saw nothing: zeros
        } else if (live) {
          float4* to_part = reinterpret_cast<float4*>(a.part_o + mine_at * HD + d);
#pragma unroll
          for (int i = 0; i < 4; ++i) to_part[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&st.o_free);
      if (!whole) {   // the pair goes on in other CTAs: the last of them to finish joins all parts, in order
        if (live && d_begin == 0) a.part_ml[mine_at] = make_float2(top, sum);
        __threadfence();
        named_bar_sync(1, 256);
        if (threadIdx.x == 0) {
          st.last = atomicAdd(a.tickets + i0, 1) == i1 - i0;
          if (st.last) a.tickets[i0] = 0;
        }
        named_bar_sync(1, 256);
        if (st.last && live) {
          __threadfence();
          auto at = [&](int i) { return static_cast<int64_t>(i == i0 ? 2 * i + 1 : 2 * i) * (2 * kRows) + slot_row; };
          float best = -INFINITY;
          sum = 0.f;
          for (int i = i0; i <= i1; ++i) best = fmaxf(best, __ldcg(a.part_ml + at(i)).x);
          for (int i = i0; i <= i1; ++i) {
            const float2 ml = __ldcg(a.part_ml + at(i));
            sum += ml.y * factor(ml, best);
          }
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll 1
          for (int d = d_begin; d < d_end; d += 16) {
            float o[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = 0.f;
#pragma unroll 2
            for (int i = i0; i <= i1; ++i) {
              const float f = factor(__ldcg(a.part_ml + at(i)), best);
              const float4* src = reinterpret_cast<const float4*>(a.part_o + at(i) * HD + d);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float4 v = __ldcg(src + k);
                o[4 * k] += v.x * f;
                o[4 * k + 1] += v.y * f;
                o[4 * k + 2] += v.z * f;
                o[4 * k + 3] += v.w * f;
              }
            }
            put(d, o, inv);
          }
        }
      }
      named_bar_sync(1, 256);   // the states (and st.last) are read before the next part's are written
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 13) {
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
  if (encode_pool_map_tc(encode, &map, c.pages, c.n_pages, c.n_kv_heads, c.head_dim) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  return c.head_dim == 128 ? launch<128, false>(a, map, ctas, stream) : launch<64, false>(a, map, ctas, stream);
}

}  // namespace kvprm
