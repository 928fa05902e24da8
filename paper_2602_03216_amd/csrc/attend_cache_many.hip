// Attention over the paged cache for sequences with many rows (prompts and pieces of them): what has to be computed bounds it.
//
// One workgroup = 128 rows of one sequence and KV head (rows of the group's heads side by side: row r is token r / g, head r % g), four
// wavefronts of 32 rows, two workgroups per CU; 64 keys per tile.  Both products on v_mfma_f32_32x32x16_bf16 in the transposed
// orientation (S^T = K Q^T, O^T = V^T P^T), as in attend.hip: a lane owns one row, and the probabilities it has are the second product's operand.
//   Unlike there V is taken as the pages have it, one row per key.  The tile goes to LDS like K's and is transposed by the reads
// (ds_read_b64_tr_b16: four keys of one column per lane, two reads per operand); the keys of an operand are then those of the accumulator's
// registers, 4 hi .. 4 hi + 3 and 8 more of every 16, in groups of four, and K's rows need no permutation.
//   A wavefront stages the 16 keys of one block of a tile, which lie on one page: one look-up per tile and wavefront, a tile ahead, out of a
// register that holds the ids of 64 blocks.  8-bit rows pass the registers, where the conversion widens them to bf16 with their power of two
// (exact): 32 conversions per wavefront and tile beside 32 products; the loop is then the same.
//   Where the row tiles of a call do not fill the chip their keys are cut into parts, joined by a second launch.
#include "attend_cache_few.h"

namespace tsa {

using namespace cache_detail;
using namespace attend_cache_detail;

namespace {

constexpr int NW = 4;
constexpr int kRowsPerWave = 32;

template <int D, bool E4M3>
struct Tiles {
  static constexpr int RB = E4M3 ? D : 2 * D, ROWB = 2 * D;       // bytes of a row in the pool, in LDS
  using KRows = LdsRows<ROWB>;
  static constexpr int RPB = KRows::RPB, LPR = KRows::LPR;         // rows of a KiB in LDS, 16-byte pieces of a row
  static constexpr int KHALF = 32 / RPB * kBlock, VTILE = kTile * ROWB;
  static constexpr int NS = D / 16, ND = D / 32;
  static constexpr int KPW = kTile / NW;                           // keys that a wavefront stages
  static constexpr int CH = KPW / RPB;                             // loads of a KiB (bf16)
  static constexpr int LPR8 = D / 16, RPL8 = 64 / LPR8, CH8 = KPW / RPL8 > 0 ? KPW / RPL8 : 1;     // 8 bits: lanes per row, rows per load, loads
  static_assert(KPW == 16, "a wavefront's keys are one block of 16");

  // V: 16-byte piece p of row r sits at p ^ v_swizzle(r), so that the rows that one transposing read touches lie in different banks
  __device__ static __forceinline__ int v_swizzle(int r) {
    return ROWB == 256 ? ((r & 3) << 2) ^ (((r >> 2) & 1) << 1) : (((r >> 1) & 1) << 2) ^ (((r >> 2) & 1) << 1);
  }
};

// Exchange format between the loads of a tile and its place in LDS, 8 bits
template <int CH8>
struct Staged {
  u32x4 x[CH8];
  uint32_t e[CH8];
};

// FEW: the workgroups behind the first `grid` ones are shares of the sequences with few rows.
template <int D, bool E4M3, bool FEW>
__global__ __launch_bounds__(64 * NW, 2) void attend_many_rows(Args a, unsigned grid) {
  using T = Tiles<D, E4M3>;
  constexpr int NS = T::NS, ND = T::ND, RB = T::RB, ROWB = T::ROWB;
  constexpr int kRings = 5 * T::KHALF + 2 * T::VTILE;    // K in a ring of five half tiles, V of two tiles
  constexpr int kFewLds = FEW ? Shape<D, E4M3, 1>::kLds : 0;
  __shared__ __attribute__((aligned(1024))) char smem[kRings > kFewLds ? kRings : kFewLds];
  if constexpr (FEW) {
    if (blockIdx.x >= grid) {
      few_rows<D, E4M3, 1, true, false>(a, smem, blockIdx.x - grid);
      return;
    }
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lo = lane & 31, hi = lane >> 5;

  // ---- workgroup -> KV head, row tile, part.  id % 8 is the XCD: the row tiles of a head stay on one (or a few) of them, the last ones first.  All tiles' first
  // parts are in front of all second ones, so that parts that a short context does not have stand at the end: between the others they spoil the spread over
  // the CUs (2176 tokens over 6000 keys, 32 / 8 heads, a table of 131072 positions: 235 us, 218 so; without such parts no difference).
  const unsigned xcd = blockIdx.x & 7u, at = blockIdx.x >> 3;
  const unsigned rank = one(a.by_vheads.div(at)), vhead = xcd * a.vheads_per_xcd + (at - rank * a.vheads_per_xcd);
  const int h = (int)(vhead >> a.split_log2);
  const unsigned item = (rank << a.split_log2) + (vhead & ((1u << a.split_log2) - 1u));
  const int part = one(a.by_slots.div(item)), slot = a.slots - 1 - (int)(item - (unsigned)part * a.slots);
  if (part >= a.splits) return;
  const int seq = one(last_up_to(a.b.n_seqs, slot, lane, [&](int i) { return first_slot(a, i); }));
  if (seq < 0 || seq >= a.b.n_seqs) return;
  const ManyTile x = many_tile(a, seq, slot - one(first_slot(a, seq)));
  if (!x.there || part >= x.parts) return;
  const int t0 = part * x.per, t1 = min(x.tiles, t0 + x.per);

  // ---- the rows of this wavefront and of this lane
  const int pos0 = x.kv - x.q_len, wrow0 = x.row0 + kRowsPerWave * wave, row = min(wrow0 + lo, x.rows - 1), tok = (int)a.by_g.div(row);
  const int pos = pos0 + tok;
  const bool has_rows = wrow0 < x.rows;
  const int wp_min = pos0 + one(a.by_g.div(min(wrow0, x.rows - 1))), wp_max = pos0 + one(a.by_g.div(min(wrow0 + kRowsPerWave, x.rows) - 1));
  const int wsee_lo = a.window ? wp_min - a.window + 1 : 0, wall_lo = a.window ? wp_max - a.window + 1 : 0, all_lo = a.window ? x.p_max - a.window + 1 : 0;
  const float c = a.c;

  // ---- pages: lane l holds the id of the 16 keys from start + 16 (64 chunk + l) on; `missing` has a bit for every one that is not there
  auto page_ids = [&](int chunk) -> int {
    const int key = x.start + 16 * (64 * chunk + lane);
    return key < x.see_hi ? a.b.page(seq, key) : -1;
  };
  int chunk = t0 >> 4, ids = page_ids(chunk), ids_next = page_ids(chunk + 1);
  unsigned long long missing = __builtin_amdgcn_ballot_w64(ids < 0);
  // place in the pools of this wavefront's block of tile t (tiles in order), and the four blocks of the tile that are not there
  auto look_up = [&](int t, int& gone) -> long long {
    if ((t >> 4) != chunk) {
      ++chunk;
      ids = ids_next;
      missing = __builtin_amdgcn_ballot_w64(ids < 0);
      ids_next = page_ids(chunk + 1);
    }
    gone = (int)(missing >> ((4 * t) & 63)) & 15;
    const int id = __builtin_amdgcn_readlane(ids, (4 * t + wave) & 63);
    return a.b.row(max(id, 0), h, x.start + kTile * t + 16 * wave);
  };

  // ---- staging
  const int lds0 = (int)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int k_part = ((16 * wave) % 32) / T::RPB * kBlock, v_part = 16 * wave * ROWB;
  const bool k_half = wave >= 2;
  const int k_off = (lane / T::LPR) * RB + 16 * T::KRows::piece(lane);
  int v_off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) v_off[i] = (lane / T::LPR) * RB + 16 * ((lane % T::LPR) ^ T::v_swizzle(i * T::RPB + lane / T::LPR));
  Staged<T::CH8> sk, sv;
  const int r8 = lane / T::LPR8, p8 = lane % T::LPR8;
  // a KiB of consecutive cached rows
  auto load_block = [&](const char* base, int off, int lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    lds = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds), "v"(off), "s"(base) : "memory");
#endif
  };
  auto load_staged = [&](Staged<T::CH8>& s, const char* pool, const uint8_t* scales, long long r) {
#pragma unroll
    for (int i = 0; i < T::CH8; ++i) {
      s.x[i] = *(const u32x4*)(pool + (r + i * T::RPL8 + r8) * RB + 16 * p8);
      s.e[i] = scales[r + i * T::RPL8 + r8];
    }
  };
  auto load_k_block = [&](long long r, int half0, int half1, int i) {
    load_block(a.kp + r * RB + i * 1024, k_off, lds0 + (k_half ? half1 : half0) + k_part + i * kBlock);
  };
  auto load_v_block = [&](long long r, int tile, int i) { load_block(a.vp + r * RB + i * 1024, v_off[i & 1], lds0 + tile + v_part + i * 1024); };
  // rows that nobody sees read as zeros: they may never have been written
  auto load_v_seen = [&](long long r, int t, int gone, int tile) {
    const int key0 = x.start + kTile * t + 16 * wave;
    const bool here = !((gone >> wave) & 1);
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < T::CH8; ++i) {
        const int key = key0 + i * T::RPL8 + r8;
        const bool seen = here && key >= x.see_lo && key < x.see_hi;
        sv.x[i] = u32x4{0, 0, 0, 0};
        sv.e[i] = 127;
        if (seen) {
          sv.x[i] = *(const u32x4*)(a.vp + (r + i * T::RPL8 + r8) * RB + 16 * p8);
          sv.e[i] = a.vs[r + i * T::RPL8 + r8];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < T::CH; ++i) {
        const int key = key0 + i * T::RPB + lane / T::LPR;
        const bool seen = here && key >= x.see_lo && key < x.see_hi;
        const char* src = seen ? a.vp + (r + i * T::RPB) * RB + v_off[i & 1] : (const char*)g_zeros + 16 * (lane % T::LPR);
        load_row_to_lds(src, lds0 + tile + v_part + i * 1024);
      }
    }
  };
  auto put8 = [&](const u32x4& w, uint32_t e, char* row_at, int sw) {
    const float s = exponent_value(e);
    *(bf16x8*)(row_at + (((2 * p8) ^ sw) << 4)) = widen8(w[0], w[1], s);
    *(bf16x8*)(row_at + (((2 * p8 + 1) ^ sw) << 4)) = widen8(w[2], w[3], s);
  };
  auto put_k = [&](int half0, int half1) {
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < T::CH8; ++i) {
        const int r = (16 * wave) % 32 + i * T::RPL8 + r8;
        put8(sk.x[i], sk.e[i], smem + (k_half ? half1 : half0) + (r / T::RPB) * kBlock + (r % T::RPB) * ROWB, T::KRows::swizzle(r));
      }
    }
  };
  auto put_v = [&](int tile) {
    if constexpr (E4M3) {
#pragma unroll
      for (int i = 0; i < T::CH8; ++i) {
        const int r = 16 * wave + i * T::RPL8 + r8;
        put8(sv.x[i], sv.e[i], smem + tile + r * ROWB, T::v_swizzle(r));
      }
    }
  };
  auto load_k = [&](long long r, int half0, int half1) {
    if constexpr (E4M3) {
      load_staged(sk, a.kp, a.ks, r);
    } else {
#pragma unroll
      for (int i = 0; i < T::CH; ++i) load_k_block(r, half0, half1, i);
    }
  };

  // ---- fragments
  int k_rd[2], v_rd[ND];
  k_rd[0] = T::KRows::read_base(lo, hi);
  k_rd[1] = k_rd[0] ^ 32;
  {
    const int i16 = lane & 15, r = 4 * hi + (i16 >> 2), piece = 2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) v_rd[dt] = r * ROWB + (((piece + 4 * dt) ^ T::v_swizzle(r)) << 4) + 8 * (i16 & 1);
  }
  auto k_frag = [&](int half, int i) -> bf16x8 { return *(const bf16x8*)(smem + half + T::KRows::read_off(k_rd, i)); };
  // 16 keys from 16 hf on, columns 32 dt ..
  auto v_frag = [&](int tile, int hf, int dt) -> bf16x8 {
    const char* p = smem + tile + v_rd[dt] + 16 * hf * ROWB;
    const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)p);
    const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(p + 8 * ROWB));
    return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  f32x16 o[1][ND], sA[1], sB[1];
  float m[1] = {kNone}, l[1] = {0.f};
  uint32_t pA[1][8], pB[1][8];
  bf16x8 qf[NS];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) o[0][dt] = f32x16{0};

  auto qk = [&](int half, f32x16& s) {
    s = f32x16{0};
#pragma unroll
    for (int i = 0; i < NS; ++i) s = mfma32(k_frag(half, i), qf[i], s);
  };
  auto pv = [&](int tile, int half, const uint32_t (&pb)[8]) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[0][dt] = mfma32(v_frag(tile, 2 * half + hf, dt), attend_detail::p_operand(pb, hf), o[0][dt]);
  };
  // S^T of half `half` of tile t in register r: key 32 half + c_row(r, hi); gone: the tile's blocks that are not there
  auto mask = [&](f32x16& s, int t, int half, int gone) {
    const int key0 = x.start + kTile * t + 32 * half, g2 = (gone >> (2 * half)) & 3;
    if (key0 + 31 <= wp_min && key0 >= wall_lo && g2 == 0) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = key0 + c_row(r, hi);
      if (((g2 >> (r >> 3)) & 1) || key > pos || (a.window && key <= pos - a.window)) s[r] = -INFINITY;
    }
  };

  // ring slots: K(t) second half in kr[0], K(t + 1) in kr[1], kr[2]; K(t + 2) goes to kr[3], kr[4]; V(t) in vc, V(t + 1) goes to vn
  int kr[5], vc = 5 * T::KHALF, vn = vc + T::VTILE;
#pragma unroll
  for (int j = 0; j < 5; ++j) kr[j] = j * T::KHALF;
  auto rotate = [&]() {
    const int x0 = kr[0], x1 = kr[1], v0 = vc;
    kr[0] = kr[2]; kr[1] = kr[3]; kr[2] = kr[4]; kr[3] = x0; kr[4] = x1;
    vc = vn; vn = v0;
  };
  auto active = [&](int t) -> bool {
    const int k0 = x.start + kTile * t;
    return t < t1 && has_rows && k0 <= wp_max && k0 + kTile - 1 >= wsee_lo;
  };
  // all rows of the workgroup see all keys of the tile
  auto full = [&](int t, int gone) -> bool {
    const int k0 = x.start + kTile * t;
    return t < t1 && k0 + kTile - 1 <= x.p_min && k0 >= all_lo && gone == 0;
  };

  // ---- prologue (tiles behind the last one: loaded from wherever the table or page 0 says, never used)
  int g0, g1, g2;
  const long long r0 = look_up(t0, g0);
  long long r1 = look_up(t0 + 1, g1), r2 = look_up(t0 + 2, g2);
  if (t0 < t1) {
    load_k(r0, kr[3], kr[0]);
    const __bf16* src = a.Q + (x.q0 + tok) * a.q_t + (h * a.g + row - tok * a.g) * a.q_h + 8 * hi;
#pragma unroll
    for (int i = 0; i < NS; ++i) qf[i] = *(const bf16x8*)(src + 16 * i);
    put_k(kr[3], kr[0]);
    load_k(r1, kr[1], kr[2]);
    put_k(kr[1], kr[2]);
    load_v_seen(r0, t0, g0, vc);
    put_v(vc);
    wait_loads();
    lds_barrier();
    qk(kr[3], sA[0]);
    lds_barrier();                                       // that slot is written in the first iteration
    if (active(t0)) {
      mask(sA[0], t0, 0, g0);
      attend_detail::softmax_max<ND, 1>(sA, c, m, l, o);
    }
  }

  // ---- the pipelined iteration: a tile that all rows of the workgroup see in full, as they do the one after it.  Same stream of chunks as in
  // attend.hip: one product and the vector work beside it that does not depend on it, fragments three chunks ahead through a ring of four.
  //    0 ..  7  S^T(t, half 1)         with  exp of half 0 (sA)
  //    8 .. 15  O^T += (t, half 0)     with  s c - m and the row max of half 1      [then the rare raise of m]
  //   16 .. 23  S^T(t + 1, half 0)     with  exp of half 1 (sB)
  //   24 .. 31  O^T += (t, half 1)     with  s c - m and the row max of (t + 1, half 0)   [wait, barrier, rare raise of m]
  constexpr int kAhead = 3, kRing = 4, kChunks = 4 * NS, CPB = NS;
  static_assert(NS == 8 || NS == 4, "the stream is laid out for d = 128 or 64");
  bf16x8 fr[kRing];
  auto fetch = [&](int k, int half1, int next0, int v_tile) {
    const int blk = k / CPB, i = k % CPB;
    if (blk == 0) fr[k % kRing] = k_frag(half1, i);
    else if (blk == 2) fr[k % kRing] = k_frag(next0, i);
    else fr[k % kRing] = v_frag(v_tile, (blk == 3 ? 2 : 0) + i / ND, i % ND);
  };
  auto fast_iter = [&]() {
    float mx = 0.f, ps0 = 0.f, ps1 = 0.f, mxc[1];
    f32x16 acc;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      const int blk = k / CPB, i = k % CPB;
      if (i == 0) {                                      // the blocks with exponentials go first (see attend.hip)
        if (blk == 0 || blk == 2) __builtin_amdgcn_s_setprio(2);
        else __builtin_amdgcn_s_setprio(0);
      }
      if (k + kAhead < kChunks) fetch(k + kAhead, kr[0], kr[1], vc);
      else fetch(k + kAhead - kChunks, kr[2], kr[3], vn);
      if constexpr (E4M3) {
        if (k == 0) load_staged(sk, a.kp, a.ks, r2);
        if (k == 1) load_staged(sv, a.vp, a.vs, r1);
        if (k == 3 * CPB) put_k(kr[3], kr[4]);
        if (k == 3 * CPB + CPB / 2) put_v(vn);
      } else {
        if (k < T::CH) load_k_block(r2, kr[3], kr[4], k);
        else if (k < 2 * T::CH) load_v_block(r1, vn, k - T::CH);
      }
      if (blk == 0 || blk == 2) {
        const f32x16& s_in = blk == 0 ? sA[0] : sB[0];
        uint32_t (&p_out)[8] = blk == 0 ? pA[0] : pB[0];
        constexpr int EPS = 16 / NS;
        if (i == 0) acc = f32x16{0};
        acc = mfma32(fr[k % kRing], qf[i], acc);
#pragma unroll
        for (int e = 0; e < EPS; e += 2) {
          const int r = EPS * i + e;
          const float p0 = fast_exp2(s_in[r]), p1 = fast_exp2(s_in[r + 1]);
          if (r == 0) { ps0 = p0; ps1 = p1; }
          else { ps0 += p0; ps1 += p1; }
          p_out[r >> 1] = attend_detail::pack_bf16(p0, p1);
        }
        if (i == CPB - 1) {
          (blk == 0 ? sB[0] : sA[0]) = acc;
          l[0] += ps0 + ps1;
        }
      } else {
        f32x16& s_in = blk == 1 ? sB[0] : sA[0];
        const uint32_t (&pb)[8] = blk == 1 ? pA[0] : pB[0];
        constexpr int EPC = 16 / CPB;
        o[0][i % ND] = mfma32(fr[k % kRing], attend_detail::p_operand(pb, i / ND), o[0][i % ND]);
#pragma unroll
        for (int e = 0; e < EPC; ++e) s_in[EPC * i + e] = fmaf(s_in[EPC * i + e], c, -m[0]);
        if (i == 0) mx = s_in[0];
#pragma unroll
        for (int e = 0; e < EPC; e += 2) mx = __builtin_fmaxf(__builtin_fmaxf(mx, s_in[EPC * i + e]), s_in[EPC * i + e + 1]);
        if (i == CPB - 1) mxc[0] = fmaxf(mx, __shfl_xor(mx, 32));
      }
      __builtin_amdgcn_sched_barrier(0);
      if (k == 2 * CPB - 1) attend_detail::raise_max_rel<ND, 1>(mxc, m, l, o, sB);
    }
    wait_loads();
    lds_barrier();
    attend_detail::raise_max_rel<ND, 1>(mxc, m, l, o, sA);
  };

  const float inv_c = 1.0f / c;
  for (int t = t0; t < t1; ++t) {
    if (full(t, g0) && full(t + 1, g1)) {
      // (the pipelined iterations hold a half tile as s c - m)
#pragma unroll
      for (int r = 0; r < 16; ++r) sA[0][r] = fmaf(sA[0][r], c, -m[0]);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) fetch(k, kr[0], kr[1], vc);
      do {
        fast_iter();
        r1 = r2;
        g0 = g1; g1 = g2;
        r2 = look_up(t + 3, g2);
        rotate();
        ++t;
      } while (full(t, g0) && full(t + 1, g1));
#pragma unroll
      for (int r = 0; r < 16; ++r) sA[0][r] = (sA[0][r] + m[0]) * inv_c;
    }
    load_k(r2, kr[3], kr[4]);
    load_v_seen(r1, t + 1, g1, vn);
    int g3;
    const long long r3 = look_up(t + 3, g3);
    if (active(t)) {
      const bool second = x.start + kTile * t + 32 <= wp_max;
      if (second) qk(kr[0], sB[0]);
      attend_detail::softmax_exp<1>(sA, c, m, l, pA);
      pv(vc, 0, pA[0]);
      if (second) {
        mask(sB[0], t, 1, g0);
        attend_detail::softmax_max<ND, 1>(sB, c, m, l, o);
        attend_detail::softmax_exp<1>(sB, c, m, l, pB);
        pv(vc, 1, pB[0]);
      }
    }
    if (active(t + 1)) {
      qk(kr[1], sA[0]);
      mask(sA[0], t + 1, 0, g1);
      attend_detail::softmax_max<ND, 1>(sA, c, m, l, o);
    }
    put_k(kr[3], kr[4]);
    put_v(vn);
    wait_loads();
    lds_barrier();
    r1 = r2; r2 = r3;
    g0 = g1; g1 = g2; g2 = g3;
    rotate();
  }

  // ---- the rows leave
  if (!has_rows) return;
  const float lt = l[0] + __shfl_xor(l[0], 32);
  if (x.parts > 1) {
    const long long first = (((long long)slot * a.b.Hkv + h) * a.splits + part) * kManyRows + kRowsPerWave * wave + lo;
    if (wrow0 + lo < x.rows) {
      float* dst = a.many_o + first * D + 4 * hi;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4*)(dst + 32 * dt + 8 * q) = f32x4{o[0][dt][4 * q], o[0][dt][4 * q + 1], o[0][dt][4 * q + 2], o[0][dt][4 * q + 3]};
      if (hi == 0) {
        a.many_ml[2 * first] = m[0];
        a.many_ml[2 * first + 1] = lt;
      }
    }
    return;
  }
  using Out = attend_detail::RowOut<D, ND, false>;
  static_assert(NW * Out::kLds <= kRings, "the rows of all wavefronts fit the tile rings");
  char* const lds_out = smem + wave * Out::kLds;
  Out out;
  out.put(o[0], lt > 0.f ? 1.0f / lt : 0.f, lds_out, lane);
#pragma unroll
  for (int j = 0; j < Out::N; ++j) {
    const int r = wrow0 + j * Out::RPI + lane / Out::LPR;
    if (r < x.rows) {
      const int tk = (int)a.by_g.div(r);
      *(u32x4*)(a.O + (x.q0 + tk) * a.o_t + (h * a.g + r - tk * a.g) * a.o_h + 8 * (lane % Out::LPR)) =
          *(const u32x4*)(lds_out + (j * Out::RPI + lane / Out::LPR) * Out::RS + 16 * (lane % Out::LPR));
    }
  }
  if (a.lse && hi == 0 && wrow0 + lo < x.rows)
    a.lse[(long long)(x.q0 + tok) * a.Hq + h * a.g + row - tok * a.g] = lt == 0.f ? -INFINITY : (m[0] + log2f(lt)) * kLn2;
}

}  // namespace

namespace {

template <int D, bool E4M3>
void launch_rows(const Args& a, unsigned grid, int shares, hipStream_t st) {
  if (shares) attend_many_rows<D, E4M3, true><<<grid + shares, 64 * NW, 0, st>>>(a, grid);
  else attend_many_rows<D, E4M3, false><<<grid, 64 * NW, 0, st>>>(a, grid);
}

}  // namespace

hipError_t launch_attend_many(Args& a, int d, bool e4m3, int shares, hipStream_t st) {
  // KV heads over the XCDs; where their number is no multiple of 8, every head is cut into alternating items
  int gcd = 8, log2 = 0;
  while (a.b.Hkv % gcd) { gcd >>= 1; ++log2; }
  a.split_log2 = log2;
  a.vheads_per_xcd = a.b.Hkv / gcd;
  const long long items = (long long)a.slots * a.splits, ranks = (items + (1 << log2) - 1) >> log2, grid = 8LL * a.vheads_per_xcd * ranks;
  if ((grid + shares) * 64 * NW > 0xffffffffLL) return hipErrorInvalidConfiguration;      // (Q and O would be 137 GB each)
  a.by_vheads = FastDiv((uint32_t)a.vheads_per_xcd, (uint64_t)a.vheads_per_xcd * (ranks + 1));
  a.by_slots = FastDiv((uint32_t)a.slots, (uint64_t)items + 8);
  if (d == 128) {
    if (e4m3) launch_rows<128, true>(a, (unsigned)grid, shares, st);
    else launch_rows<128, false>(a, (unsigned)grid, shares, st);
  } else {
    if (e4m3) launch_rows<64, true>(a, (unsigned)grid, shares, st);
    else launch_rows<64, false>(a, (unsigned)grid, shares, st);
  }
  return hipGetLastError();
}

}  // namespace tsa
