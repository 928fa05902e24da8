// Attention of the new tokens of a ragged batch over the paged cache:
//   o_t = sum_j softmax_j(scale q_t . k_j) v_j over the keys j of t's sequence with p_t - window < j <= p_t.
//
// The g query heads of a KV head and the new tokens of a sequence are the rows of one matrix: row r is token r / g, head r % g of
// the group, so K and V are read once for all of them.
//
// Few rows per sequence (single tokens, drafted tokens): K and V are what has to be read, HBM bounds it, and the keys are the axis that
// fills the chip.  The work of the whole batch, counted in steps of 128 keys of one (sequence, KV head, tile of 16, 32 or 64 rows), is cut into
// equal shares, one per workgroup; lengths are known on the device only, so every workgroup sums them up itself and finds its
// place.  A share that covers only a part of a row tile's keys leaves its running max, sum and output in the workspace, and a second launch
// joins them; whole ones are written at once.  Where contexts are short and few, a workgroup takes a whole tile instead (WHOLE).
//   A wavefront takes 32 keys of a step, with a softmax of its own; they meet at the end of a segment.  S^T = K Q^T on
// v_mfma_f32_16x16x32_bf16: rows = keys, columns = the tile's rows, so a lane keeps one row's max and sum.  K goes from memory straight
// into the registers of that product (a lane's 16 bytes are its operand).  O^T = V^T P^T takes the probabilities as the lane holds them: its
// contraction index runs over keys 4 q .. 4 q + 3 of the first 16 and of the second 16 keys (q = lane / 16), and V^T comes out of LDS
// by the transposing reads, four (eight in 8 bits) keys of one column per lane.  V goes to LDS without passing registers; the
// next step's K and V are in flight while a step is computed, and no wavefront waits for another inside a segment.
//   8 bits: K is widened to bf16 with its row's power of two by the conversion (exact), V without it, and V's power goes into the
// probability in front of its rounding.
#pragma once

#include "attend_cache.h"

namespace tsa {

namespace attend_cache_detail {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// What a sequence asks for.
struct Seq {
  int q0, q_len, kv, rows, tiles, first, steps;          // first: its first key that any query sees, rounded down to 16
  // steps of all its row tiles, each counted as a multiple of `of`
  __device__ __forceinline__ uint32_t units(int Hkv, int of) const { return (uint32_t)(Hkv * tiles) * span(of); }
  __device__ __forceinline__ uint32_t span(int of) const { return of == 1 ? steps : (uint32_t)((steps + of - 1) / of) * of; }
};

__device__ __forceinline__ Seq sequence(const Args& a, int q0, int q_end, int kv, int rt, int step) {
  Seq s;
  s.q0 = q0;
  s.q_len = max(q_end - q0, 0);
  s.kv = kv;
  s.rows = s.q_len * a.g;
  if (s.rows > a.few) s.rows = 0;
  s.tiles = (s.rows + rt - 1) / rt;
  s.first = a.window ? max(0, s.kv - s.q_len - a.window + 1) & ~15 : 0;
  s.steps = max(1, (s.kv - s.first + step - 1) / step);
  return s;
}

__device__ __forceinline__ Seq sequence(const Args& a, int i, int rt) { return sequence(a, a.b.first(i), a.b.first(i + 1), a.b.kv(i), rt, kStep); }
__device__ __forceinline__ Seq one_sequence(const Args& a, int i, int rt, int step) {
  Seq s = sequence(a, one(a.b.first(i)), one(a.b.first(i + 1)), one(a.b.kv(i)), rt, step);
  s.tiles = one(s.tiles);
  s.steps = one(s.steps);
  return s;
}

// Shares per CU, all of which run at once.  What they have in flight together is what the memory rate comes from: the rows of d = 64 in 8 bits
// are short and take four (300 sequences x 1000 keys, 8 KV heads: 83 us with two, 70 with four, 6 x 131072 153 and 138); with longer rows two have enough
// in flight, and more only cut the work finer (64 x 8192 in 8 bits, d = 128: 176 us with two, 189 with three; bf16, d = 64: 170 with two, 176 with four).
// (In the joint launch with prompts two workgroups a CU run at once whatever this says: d = 64 in 8 bits has its shares there in two rounds, in the launch's tail.)
constexpr int per_cu(int d, bool e4m3, int mb) { return mb == 4 && d == 128 ? 1 : mb == 1 && d == 64 && e4m3 ? 4 : 2; }

template <int D, bool E4M3, int MB, int NW = 4>
struct Shape {
  static constexpr int RT = 16 * MB;                     // rows of a tile
  static constexpr int kPerCU = per_cu(D, E4M3, MB), kShares = 256 * kPerCU;
  static constexpr int RB = E4M3 ? D : 2 * D;            // bytes of a cached row
  static constexpr int LPR = RB / 16, RPI = 64 / LPR;    // lanes per row, rows of a load into LDS
  static constexpr int NK = RB / 64;                     // 16-byte pieces of a row of K per lane
  static constexpr int NS = D / 32, ND = D / 16;         // k-steps of the first product, column tiles of the second
  static constexpr int kRing = 2 * 32 * RB;              // LDS bytes of a wavefront: two steps of V
  static constexpr int OS = D + 4;                       // floats between rows where the wavefronts meet
  static constexpr int kMerge = NW * RT * OS * 4;
  static constexpr int kTiles = NW * kRing > kMerge ? NW * kRing : kMerge;
  struct Tail {
    float ml[NW][RT][2];                                  // where the wavefronts meet: max and sum of every row
    uint32_t scan[16], place[2];
  };
  static constexpr int kLds = kTiles + (int)sizeof(Tail);
  // 16-byte piece p of row r of V is kept at p ^ swizzle(r): the 32 lanes that a transposing read serves at once then touch all banks
  __device__ static __forceinline__ int swizzle(int r) {
    if (!E4M3) return RB == 256 ? (r & 7) << 1 : ((r >> 1) & 3) << 1;
    return RB == 128 ? ((r >> 1) & 3) | ((r >> 4) & 1) << 2 : ((r >> 2) & 1) | ((r >> 4) & 1) << 1;
  }
};

// Sums of x over lanes 0 .. this one, in six additions without LDS.
__device__ __forceinline__ uint32_t sum_up_to_lane(uint32_t x) {
  const auto add = [&](uint32_t y) { x += y; };
  add(__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));       // from 1, 2, 4, 8 lanes below, inside 16
  add(__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  add(__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  add(__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  add(__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));       // lane 15 of a row into the next one, lane 31 into the upper half
  add(__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
  return x;
}
// Sums over the wavefront, or over all four of the workgroup.
template <int N>
__device__ __forceinline__ void sum_up(uint32_t (&x)[N], bool alone, uint32_t* scan, int lane, int wave) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_readlane(sum_up_to_lane(x[i]), 63);
  if (alone) return;
  __syncthreads();
  if (lane < N) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane == i) scan[4 * i + wave] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = one(scan[4 * i] + scan[4 * i + 1] + scan[4 * i + 2] + scan[4 * i + 3]);
}

// K of a step in registers, and the exponents of both.
template <int NK>
struct StepRegs {
  u32x4 k[2][NK];
  uint32_t ks[2], vs[2];
};

// Share `block` of the batch, by a workgroup of 256 threads with Shape::kLds bytes of LDS at `smem`.  ONCE: no row of K and V is read twice.
// WHOLE: by one of 512 threads that takes whole row tiles, in steps of 256 keys; `block` counts KV heads, then a.whole tiles of a sequence, then sequences.
template <int D, bool E4M3, int MB, bool ONCE, bool WHOLE>
__device__ __forceinline__ void few_rows(const Args& a, char* smem, unsigned block) {
  constexpr int NW = WHOLE ? 8 : 4, kKeys = 32 * NW, kBlocks = 2 * NW, kChunkLog2 = WHOLE ? 2 : 3;      // keys of a step, 16 of them each, steps of 64 such
  using S = Shape<D, E4M3, MB, NW>;
  constexpr int RT = S::RT, RB = S::RB, kShares = S::kShares;
  auto& tail = *(typename S::Tail*)(smem + S::kTiles);
  auto& ml = tail.ml;
  auto& scan = tail.scan;
  auto& place = tail.place;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lo = lane & 15, quarter = lane >> 4;
  const int n = a.b.n_seqs, Hkv = a.b.Hkv;
  uint32_t share = 0, u = 0, end = 0, in_seq = 0;
  int of = 1, seq = 0, whole_h = 0, whole_tile = 0;
  if constexpr (WHOLE) {
    const int rest = one((int)(block / (unsigned)Hkv));
    whole_h = (int)block - rest * Hkv;
    seq = one(rest / a.whole);
    whole_tile = rest - seq * a.whole;
    if (seq >= n) return;
  } else {
    // ---- the share: thread t counts sequences t * per .. of the batch.  Where a few steps more than an equal share let no share go over the end of
    // a row tile, the tiles are counted as multiples of such a share: another tile in a share costs a meeting of the wavefronts and a start, which is
    // about as long as three steps (9 sequences x 4096 keys, 4 KV heads, two row tiles, 8 bits: equal shares of 4.5 steps 34 us, whole ones of 5 28).
    // (Up to 64 sequences every wavefront does it for itself, a sequence per lane, without a barrier.)
    const bool alone = n <= 64;
    const int per = (n + 255) / 256, who = alone ? lane : tid, i0 = who * per, i1 = min(n, i0 + per);
    const Seq own = sequence(a, min(i0, n - 1), RT);
    const auto over_mine = [&](auto&& f) {
      for (int i = i0; i < i1; ++i) f(i, per == 1 ? own : sequence(a, i, RT));
    };
    uint32_t mine = 0, sum[1];
    over_mine([&](int, const Seq& q) { mine += q.units(Hkv, 1); });
    sum[0] = mine;
    sum_up(sum, alone, scan, lane, wave);
    share = (sum[0] + kShares - 1) / kShares;
    if (share > 1) {
      // shares that whole ones of share + k steps make; over the workgroup a sum is two barriers, so all k at once (2000 x 100 keys 109 -> 98 us)
      const auto count = [&](auto& parts, int k0) {
        over_mine([&](int, const Seq& q) {
#pragma unroll
          for (int k = 0; k < (int)(sizeof(parts) / 4); ++k) parts[k] += (uint32_t)(Hkv * q.tiles) * ((q.steps + share + k0 + k - 1) / (share + k0 + k));
        });
        sum_up(parts, alone, scan, lane, wave);
      };
      if (alone) {
        for (int k = 0; k < 4 && of == 1; ++k) {
          uint32_t parts[1] = {0};
          count(parts, k);
          if (parts[0] <= (uint32_t)kShares) of = (int)share + k;
        }
      } else {
        uint32_t parts[4] = {0, 0, 0, 0};
        count(parts, 0);
#pragma unroll
        for (int k = 3; k >= 0; --k)
          if (parts[k] <= (uint32_t)kShares) of = (int)share + k;
      }
      if (of > 1) {
        share = of;
        mine = 0;
        over_mine([&](int, const Seq& q) { mine += q.units(Hkv, of); });
      }
    }
    if (tid < 2) a.cut[2 * block + tid].parts = 0;
    uint32_t upto = sum_up_to_lane(mine), total;
    of = one(of);
    share = one(share);
    u = block * share;
    if (alone) {
      total = __builtin_amdgcn_readlane(upto, 63);
      if (u >= total) return;
      const unsigned long long behind = __builtin_amdgcn_ballot_w64(u < upto);
      if (behind == 0) return;                             // (cu_q that does not ascend)
      seq = __ffsll((long long)behind) - 1;
      in_seq = u - __builtin_amdgcn_readlane(upto - mine, seq);
    } else {
      __syncthreads();
      if (lane == 63) scan[wave] = upto;
      if (tid == 0) place[0] = n;
      __syncthreads();
      total = 0;
      for (int w = 0; w < 4; ++w) {
        if (w < wave) upto += scan[w];
        total += scan[w];
      }
      total = one(total);
      if (u >= total) return;
      uint32_t at = upto - mine;
      if (u >= at && u < upto)
        over_mine([&](int i, const Seq& q) {
          const uint32_t x = q.units(Hkv, of);
          if (u >= at && u < at + x) {
            place[0] = i;
            place[1] = u - at;
          }
          at += x;
        });
      __syncthreads();
      seq = place[0];
      in_seq = place[1];
    }
    seq = one(seq);
    in_seq = one(in_seq);
    end = u + share < total ? u + share : total;
  }

  const int lds0 = (int)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * S::kRing;
  char* const ring = smem + wave * S::kRing;
  // transposing reads: this lane's address in a step's V, up to the column tile (an exclusive or) and, in bf16, the second 16 keys
  const int v_row = E4M3 ? 4 * quarter + ((lo >> 1) & 3) + ((lo >> 3) << 4) : 4 * quarter + (lo >> 2);
  const int v_rd = v_row * RB + (E4M3 ? (S::swizzle(v_row) << 4) + 8 * (lo & 1) : ((S::swizzle(v_row) ^ ((lo >> 1) & 1)) << 4) + 8 * (lo & 1));

  Seq q;
  if constexpr (WHOLE) q = one_sequence(a, seq, RT, kKeys);
  while (WHOLE || u < end) {
    uint32_t span = 0, units = 0;
    int h = whole_h, tile = whole_tile, s0 = 0, s1 = 0;
    if constexpr (WHOLE) {
      if (tile >= q.tiles) return;
      s1 = q.steps;
    } else {
      for (;; ++seq) {
        if (seq >= n) return;                              // (cu_q that does not ascend: the sums do not hold)
        q = one_sequence(a, seq, RT, kKeys);
        if (q.tiles > 0) break;
      }
      span = one(q.span(of));
      const uint32_t ht = one(in_seq / span);
      h = one(ht / q.tiles);
      if (h >= Hkv) return;                                // (the same)
      tile = ht - h * q.tiles;
      const uint32_t in_tile = in_seq - ht * span;
      units = min(end - u, span - in_tile);
      s0 = (int)in_tile;
      s1 = min((int)(in_tile + units), q.steps);
    }

    // ---- the rows
    const int row0 = tile * RT, pos0 = q.kv - q.q_len;
    const int p_min = pos0 + one(a.by_g.div(row0)), p_max = pos0 + one(a.by_g.div(min(row0 + RT, q.rows) - 1));
    const int see_lo = a.window ? max(0, p_min - a.window + 1) : 0, see_hi = p_max + 1;     // keys that some row of the tile sees
    const int all_lo = a.window ? p_max - a.window + 1 : 0;                                 // keys all_lo .. p_min are seen by all of them
    bf16x8 qf[MB][S::NS];
    int pos[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int r = min(row0 + 16 * mb + lo, q.rows - 1), tok = (int)a.by_g.div(r);
      pos[mb] = pos0 + tok;
      const __bf16* src = a.Q + (q.q0 + tok) * a.q_t + (h * a.g + r - tok * a.g) * a.q_h;
#pragma unroll
      for (int st = 0; st < S::NS; ++st)
        qf[mb][st] = *(const bf16x8*)(src + (E4M3 ? 64 * (st >> 1) + 16 * quarter + 8 * (st & 1) : 32 * st + 8 * quarter));
    }

    // ---- pages: lane l holds the id of the 16 keys from 16 (64 chunk + l) on, counted from q.first
    auto page_ids = [&](int chunk) -> int {
      const int key = q.first + 16 * (64 * chunk + lane);
      return key < see_hi ? a.b.page(seq, key) : -1;
    };
    int chunk = s0 >> kChunkLog2, ids = page_ids(chunk), ids_next = page_ids(chunk + 1);
    auto issue = [&](int s, StepRegs<S::NK>& x, int buf) {
      if ((s >> kChunkLog2) != chunk) {
        ++chunk;
        ids = ids_next;
        ids_next = page_ids(chunk + 1);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int id = __builtin_amdgcn_readlane(ids, (kBlocks * s + 2 * wave + j) & 63);
        const int key0 = q.first + 16 * (kBlocks * s + 2 * wave + j);
        const long long row = a.b.row(max(id, 0), h, key0);
        const char* kr = a.kp + (row + lo) * RB + 16 * quarter;
#pragma unroll
        for (int i = 0; i < S::NK; ++i) x.k[j][i] = ONCE ? __builtin_nontemporal_load((const u32x4*)(kr + 64 * i)) : *(const u32x4*)(kr + 64 * i);
        if (E4M3) {
          x.ks[j] = a.ks[row + lo];
          x.vs[j] = *(const uint32_t*)(a.vs + row + 4 * quarter);
        }
#pragma unroll
        for (int i = 0; i < 16 / S::RPI; ++i) {
          const int r = i * S::RPI + lane / S::LPR, piece = (lane % S::LPR) ^ S::swizzle(16 * j + r);
          const bool seen = id >= 0 && key0 + r >= see_lo && key0 + r < see_hi;
          load_row_to_lds<ONCE>((seen ? a.vp + (row + r) * RB : (const char*)g_zeros) + 16 * piece, lds0 + buf * (32 * RB) + (16 * j + i * S::RPI) * RB);
        }
      }
    };

    f32x4 o[MB][S::ND];
    float m[MB], l[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      m[mb] = kNone;
      l[mb] = 0.f;
#pragma unroll
      for (int dt = 0; dt < S::ND; ++dt) o[mb][dt] = f32x4{0, 0, 0, 0};
    }

    auto compute = [&](int s, int ids_s, const StepRegs<S::NK>& x, int buf) {
      const int key0 = q.first + 16 * (kBlocks * s + 2 * wave);
      bool masked[2], dead[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int k0 = key0 + 16 * j;
        const bool gone = __builtin_amdgcn_readlane(ids_s, (kBlocks * s + 2 * wave + j) & 63) < 0;
        dead[j] = gone || k0 >= see_hi || k0 + 15 < see_lo;
        masked[j] = dead[j] || k0 + 15 > p_min || k0 < all_lo;
      }
      if (dead[0] && dead[1]) return;
      f32x4 sc[MB][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) sc[mb][j] = f32x4{0, 0, 0, 0};
        const float k_scale = E4M3 ? exponent_value(x.ks[j]) : 1.0f;
#pragma unroll
        for (int st = 0; st < S::NS; ++st) {
          bf16x8 kf;
          if (E4M3) kf = widen8(x.k[j][st >> 1][2 * (st & 1)], x.k[j][st >> 1][2 * (st & 1) + 1], k_scale);
          else kf = __builtin_bit_cast(bf16x8, x.k[j][st]);
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) sc[mb][j] = mfma16(kf, qf[mb][st], sc[mb][j]);
        }
        if (masked[j]) {
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int key = key0 + 16 * j + 4 * quarter + r;
              if (dead[j] || key > pos[mb] || (a.window && key <= pos[mb] - a.window)) sc[mb][j][r] = -INFINITY;
            }
        }
      }
      // (8 bits: asked for in front of the softmax; verification of 8 tokens x 32 sequences 114 -> 112 us.  In bf16 that holds too many registers: 183 -> 203.)
      typedef __attribute__((ext_vector_type(2))) int i32x2;
      i32x2 v8[S::ND];
      if constexpr (E4M3) {
#pragma unroll
        for (int dt = 0; dt < S::ND; ++dt)
          v8[dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(ring + buf * (32 * RB) + (v_rd ^ (dt << 4))));
        __builtin_amdgcn_sched_barrier(0);
      }
      bf16x8 pf[MB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        float mx = sc[mb][0][0];
#pragma unroll
        for (int r = 1; r < 8; ++r) mx = fmaxf(mx, sc[mb][r >> 2][r & 3]);
        mx *= a.c;
        if (__any(mx > m[mb] + kLag)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float mn = fmaxf(m[mb], mx), alpha = fast_exp2(m[mb] - mn);
          m[mb] = mn;
          l[mb] *= alpha;
#pragma unroll
          for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[mb][dt][r] *= alpha;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = fast_exp2(fmaf(sc[mb][j][r], a.c, -m[mb]));
            l[mb] += p;
            // (bf16 for the product, as the other attention kernels have it; V's power of two is exact.  A byte of a row that nobody
            // has written may say infinity, next to a probability of 0.)
            pf[mb][4 * j + r] = (__bf16)(E4M3 ? p * fminf(exponent_value((x.vs[j] >> (8 * r)) & 0xffu), 0x1p127f) : p);
          }
      }
#pragma unroll
      for (int dt = 0; dt < S::ND; ++dt) {
        bf16x8 vf;
        if constexpr (E4M3) {
          vf = widen8((uint32_t)v8[dt][0], (uint32_t)v8[dt][1], 1.0f);
        } else {
          const char* at = ring + buf * (32 * RB) + (v_rd ^ (dt << 5));
          const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)at);
          const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(at + 16 * RB));
          vf = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) o[mb][dt] = mfma16(vf, pf[mb], o[mb][dt]);
      }
    };

    StepRegs<S::NK> xa, xb;
    issue(s0, xa, 0);
    for (int s = s0;; s += 2) {
      wait_all();
      int ids_s = ids;
      if (s + 1 < s1) issue(s + 1, xb, 1);
      compute(s, ids_s, xa, 0);
      if (s + 1 >= s1) break;
      wait_all();
      ids_s = ids;
      if (s + 2 < s1) issue(s + 2, xa, 0);
      compute(s + 1, ids_s, xb, 1);
      if (s + 2 >= s1) break;
    }

    // ---- the wavefronts meet
    const auto max_of = [&](int r) {
      float mt = ml[0][r][0];
#pragma unroll
      for (int w = 1; w < NW; ++w) mt = fmaxf(mt, ml[w][r][0]);
      return mt;
    };
    __syncthreads();                                     // (the rings are free)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      l[mb] += __shfl_xor(l[mb], 16);
      l[mb] += __shfl_xor(l[mb], 32);
      if (quarter == 0) {
        ml[wave][16 * mb + lo][0] = m[mb];
        ml[wave][16 * mb + lo][1] = l[mb];
      }
    }
    __syncthreads();
    float* const meet = (float*)smem;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int r = 16 * mb + lo;
      const float mt = max_of(r), alpha = fast_exp2(m[mb] - mt);
#pragma unroll
      for (int dt = 0; dt < S::ND; ++dt) *(f32x4*)(meet + (wave * RT + r) * S::OS + 16 * dt + 4 * quarter) = o[mb][dt] * alpha;
    }
    __syncthreads();
    const bool complete = WHOLE || (s0 == 0 && s1 == q.steps);
    const int side = s0 == 0 ? 1 : 0;
    if (!complete && tid == side) {
      const uint32_t begin = u - s0, first = begin / share;
      a.cut[2 * block + side] = Cut{(int)((begin + q.steps - 1) / share - first) + 1, (int)(block - first), q.q0, h, row0, min(RT, q.rows - row0)};
    }
    const long long slot = 2LL * block + side;
    for (int task = tid; task < RT * (D / 8); task += 64 * NW) {
      const int r = task / (D / 8), col = 8 * (task % (D / 8));
      if (row0 + r >= q.rows) continue;
      const float mt = max_of(r);
      float lt = 0.f;
      f32x4 v[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        lt += ml[w][r][1] * fast_exp2(ml[w][r][0] - mt);
        v[0] += *(const f32x4*)(meet + (w * RT + r) * S::OS + col);
        v[1] += *(const f32x4*)(meet + (w * RT + r) * S::OS + col + 4);
      }
      if (complete) {
        const int tok = (int)a.by_g.div(row0 + r), head = h * a.g + row0 + r - tok * a.g;
        const float inv = lt > 0.f ? 1.0f / lt : 0.f;
        bf16x8 out;
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (__bf16)(v[i >> 2][i & 3] * inv);
        *(bf16x8*)(a.O + (q.q0 + tok) * a.o_t + head * a.o_h + col) = out;
        if (a.lse && col == 0) a.lse[(long long)(q.q0 + tok) * a.Hq + head] = lt == 0.f ? -INFINITY : (mt + log2f(lt)) * kLn2;
      } else {
        float* dst = a.part_o + (slot * RT + r) * D + col;
        *(f32x4*)dst = v[0];
        *(f32x4*)(dst + 4) = v[1];
        if (col == 0) {
          a.part_ml[(slot * RT + r) * 2] = mt;
          a.part_ml[(slot * RT + r) * 2 + 1] = lt;
        }
      }
    }
    __syncthreads();
    if constexpr (WHOLE) {
      whole_tile += a.whole;
    } else {
      u += units;
      in_seq += units;
      if (in_seq >= (uint32_t)(Hkv * q.tiles) * span) {
        ++seq;
        in_seq = 0;
      }
    }
  }
}

}  // namespace attend_cache_detail

}  // namespace tsa
