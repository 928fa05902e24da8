// Pieces shared by the two ways of the attention over the paged cache (attend_cache.hip: sequences with few rows, and the joining of parts;
// attend_cache_many.hip: sequences with many rows).
#pragma once

#include "attend_common.h"
#include "cache_common.h"

namespace tsa {

using namespace cache_detail;
using attend_detail::kBlock;
using attend_detail::lds_barrier;
using attend_detail::LdsRows;
using attend_detail::wait_loads;

namespace attend_cache_detail {

constexpr float kNone = attend_detail::kNegBig;          // running max of a row that has seen no key
constexpr float kLag = attend_detail::kLazy;             // log2 units that the running max may lag behind
constexpr int kStep = 128;                               // keys of a step
constexpr int kTile = 64;                                // many rows: keys of a tile
constexpr int kPartTiles = 8;                            // ... and fewest tiles of a part
constexpr int kManyRows = 128;                           // ... and rows of a workgroup
constexpr int kFewRows = 64;                             // sequences of at most so many rows (new tokens times heads of a group) are dealt by keys, the others by rows

// A row tile of which a share has a part only: its parts (0: there is none), which one the share has, and the tile's rows.
struct Cut {
  int parts, part, q0, head, row0, rows;
};

struct Args {
  Batch b;
  const __bf16* Q;
  const char* kp;
  const char* vp;
  const uint8_t* ks;
  const uint8_t* vs;
  __bf16* O;
  float* lse;
  long long q_t, q_h, o_t, o_h;
  int Hq, g, window;
  float c;                       // scale * log2(e)
  FastDiv by_g;
  // workspace
  Cut* cut;                      // [shares][2]: the one that a share begins in the midst of, the one that it ends in the midst of
  float* part_o;                 // [2 shares][rt][d]
  float* part_ml;                // [2 shares][rt][2]
  int rt, shares, whole;         // rows of a tile; whole tiles of a sequence that run side by side
  // sequences of more rows than `few` go the way of many rows: 128 of them per workgroup, a tile's keys in up to `splits` parts, or `short_splits`
  // where the sequence's new tokens see fewer than `long_keys` keys
  int few, splits, short_splits, long_keys, slots, by_rows;      // (by_rows: which slots a sequence has, see first_slot)
  float* many_o;                 // [slots][Hkv][splits][128][d]
  float* many_ml;                // [slots][Hkv][splits][128][2]
  int split_log2, vheads_per_xcd;
  FastDiv by_vheads, by_slots;
};

// The same in all lanes, and kept in a scalar: the compiler forms quotients, and what is loaded or shuffled, in vector registers, and leaves everything
// that follows from them there: addresses, loop counts and branches, some thirty registers of a kernel.
__device__ __forceinline__ int one(int x) { return __builtin_amdgcn_readfirstlane(x); }

// 64 lanes' 16 bytes to LDS bytes lds .. lds + 1023.  Counted by vmcnt and by nothing that the compiler tracks; no output register.  The wait
// states: m0 may come out of a vector instruction.  ONCE: the bytes are not kept in the caches.
template <bool ONCE = false>
__device__ __forceinline__ void load_row_to_lds(const void* p, int lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  lds = __builtin_amdgcn_readfirstlane(lds);
  if (ONCE) asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, off nt" ::"{m0}"(lds), "v"(p) : "memory");
  else asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(lds), "v"(p) : "memory");
#endif
}
// Everything that this wavefront asked for has landed, in registers and in LDS, and its LDS reads are done.
__device__ __forceinline__ void wait_all() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  u32x4 w;
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return __builtin_bit_cast(bf16x8, w);
}

__device__ const u32x4 g_zeros[16] = {};                 // a row of V for keys that nobody sees

// Many rows: what the workgroups of one row tile (128 rows of one sequence and KV head) have in common.
struct ManyTile {
  int q0, q_len, kv, rows, row0;
  int p_min, p_max;              // positions of its first and last row
  int see_lo, see_hi;            // keys see_lo .. see_hi - 1 are seen by some row
  int start, tiles;              // key tiles: start, start + 64, ..
  int per, parts;                // tiles of a part, parts
  bool there;
};
__device__ __forceinline__ ManyTile many_tile(const Args& a, int seq, int tile) {
  ManyTile x;
  x.q0 = one(a.b.first(seq));
  x.q_len = max(one(a.b.first(seq + 1)) - x.q0, 0);
  x.kv = one(a.b.kv(seq));
  x.rows = x.q_len * a.g;
  x.row0 = tile * kManyRows;
  x.there = tile >= 0 && x.rows > a.few && x.row0 < x.rows;      // (tile < 0: cu_q that does not ascend)
  const int pos0 = x.kv - x.q_len;
  x.p_min = pos0 + one(a.by_g.div(max(0, min(x.row0, x.rows - 1))));
  x.p_max = pos0 + one(a.by_g.div(max(0, min(x.row0 + kManyRows, x.rows) - 1)));
  x.see_lo = a.window ? max(0, x.p_min - a.window + 1) : 0;
  x.see_hi = x.p_max + 1;
  x.start = x.see_lo & ~15;
  x.tiles = max(0, (x.see_hi - x.start + kTile - 1) / kTile);
  const int seen = a.window ? min(x.kv, a.window + x.q_len) : x.kv;
  const int parts = max(1, min(seen < a.long_keys ? a.short_splits : a.splits, x.tiles / kPartTiles));
  x.per = one((x.tiles + parts - 1) / parts);
  x.parts = one(x.per ? (x.tiles + x.per - 1) / x.per : 1);
  return x;
}
// First slot of a sequence's row tiles in the grid and in the workspace, from the rows x in front of it alone (a sum over the batch would be in front of
// every workgroup's first load).  Either x in tiles and one more for every sequence: right for all, and most of it empty where many sequences
// have few rows.  Or x / 64.5: a sequence of r > 64 rows has ceil(r / 128) tiles, never more than floor(2 r / 129), so it reaches no slot of the next one;
// sequences with fewer rows have none.  The host takes what needs fewer slots: 64 single tokens of a caller who does not know that they are single have
// 3 slots a head instead of 66, and their parts 60 MB instead of 1.1 GB.
static_assert(kManyRows == 2 * kFewRows, "2 r / (kManyRows + 1) holds the tiles of r > kFewRows rows");
__device__ __forceinline__ int first_slot(const Args& a, int seq) {
  const int rows = a.b.first(seq) * a.g;                 // (at most 2^30)
  return a.by_rows ? (int)(2u * (unsigned)rows / (kManyRows + 1)) : rows / kManyRows + seq;
}

}  // namespace attend_cache_detail

// attend_cache_many.hip: sets the grid's part of the arguments
// shares: workgroups for the sequences with few rows (tiles of 16) in the same launch, or 0
hipError_t launch_attend_many(attend_cache_detail::Args& a, int d, bool e4m3, int shares, hipStream_t st);

}  // namespace tsa
