// Rotary positions: the pair (x, y) of columns that belongs to frequency f, of a row at position p, becomes
//   gain * (x cos a - y sin a,  x sin a + y cos a),   a = p f.
// Every element is read once and written once: HBM bounds it.
//
// Angles.  A position of a million times a frequency of one radian leaves 32-bit floats some 0.06 rad, so the angle is never
// formed in radians: the host hands each frequency over in turns per position as a 64-bit fraction (2^64 = one turn), the
// product with the position wraps around modulo one turn by itself, exactly, and its top 32 bits are the angle to 2^-32 of a
// turn, as a 32-bit float within 2^-25.  sin and cos are those of the 32-bit library on half turns in [-1, 1].
//
// A thread owns eight pairs (two 16-byte pieces of a row: one from either half, or 32 consecutive bytes where the pairs
// lie side by side) of one token, and takes them through the heads: sines and cosines are formed once per token, not once per
// head.  Eight adjacent lanes (four at d = 64) cover a row; the rest of a row's columns, which are not rotated, travels as
// units of the same size.
#include "tsa_internal.h"

namespace tsa {

namespace {

struct RotaryKernelArgs {
  const __bf16* Q;
  const __bf16* K;
  __bf16* Qo;
  __bf16* Ko;
  const int32_t* positions;
  Strides q, k, qo, ko;
  long long rows;                // B * L tokens
  int Hq, heads, L, units, rot_units, half, start;
  float gain;
  FastDiv by_L;
  uint64_t turns[kRotaryFreqs];
};

__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t round_pair(float lo, float hi) {
  bf16x2 v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}

// UN units per row (d / 16), 1 << tt_log2 tokens per workgroup; the other 256 / (UN << tt_log2) threads take other heads.
template <bool INTERLEAVED, int UN>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryKernelArgs a, int tt_log2, unsigned first) {
  constexpr int UN_LOG2 = UN == 8 ? 3 : 2, kBatch = 2;
  const int tid = threadIdx.x, u = tid & (UN - 1);
  const int tok = (tid >> UN_LOG2) & ((1 << tt_log2) - 1), lane_head = tid >> (UN_LOG2 + tt_log2), step = 256 >> (UN_LOG2 + tt_log2);
  const long long row = ((long long)(blockIdx.x + first) << tt_log2) + tok;
  if (row >= a.rows) return;
  const uint32_t b = a.by_L.div((uint32_t)row), t = (uint32_t)row - b * (uint32_t)a.L;
  const bool rotated = u < a.rot_units;
  // columns of the unit's two pieces
  const int col0 = INTERLEAVED || !rotated ? 16 * u : 8 * u, col1 = INTERLEAVED || !rotated ? col0 + 8 : col0 + a.half;
  float cs[8], sn[8];
  if (rotated) {
    const int p = a.positions ? a.positions[row] : a.start + (int)t;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint64_t phase = (uint64_t)(long long)p * a.turns[8 * u + i];
      const float half_turns = (float)(int32_t)(phase >> 32) * 0x1p-31f;
      sincospif(half_turns, &sn[i], &cs[i]);
      sn[i] *= a.gain;
      cs[i] *= a.gain;
    }
  }
  for (int h0 = lane_head; h0 < a.heads; h0 += kBatch * step) {
    u32x4 x[kBatch], y[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * step;
      if (h < a.heads) {
        const __bf16* src = h < a.Hq ? a.Q + a.q.head(b, h) + t * a.q.l : a.K + a.k.head(b, h - a.Hq) + t * a.k.l;
        x[j] = __builtin_nontemporal_load((const u32x4*)(src + col0));
        y[j] = __builtin_nontemporal_load((const u32x4*)(src + col1));
      }
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * step;
      if (h < a.heads) {
        if (rotated) {
          if (INTERLEAVED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x0 = lo_f32(x[j][i]), y0 = hi_f32(x[j][i]), x1 = lo_f32(y[j][i]), y1 = hi_f32(y[j][i]);
              x[j][i] = round_pair(x0 * cs[i] - y0 * sn[i], x0 * sn[i] + y0 * cs[i]);
              y[j][i] = round_pair(x1 * cs[4 + i] - y1 * sn[4 + i], x1 * sn[4 + i] + y1 * cs[4 + i]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x0 = lo_f32(x[j][i]), x1 = hi_f32(x[j][i]), y0 = lo_f32(y[j][i]), y1 = hi_f32(y[j][i]);
              x[j][i] = round_pair(x0 * cs[2 * i] - y0 * sn[2 * i], x1 * cs[2 * i + 1] - y1 * sn[2 * i + 1]);
              y[j][i] = round_pair(x0 * sn[2 * i] + y0 * cs[2 * i], x1 * sn[2 * i + 1] + y1 * cs[2 * i + 1]);
            }
          }
        }
        __bf16* dst = h < a.Hq ? a.Qo + a.qo.head(b, h) + t * a.qo.l : a.Ko + a.ko.head(b, h - a.Hq) + t * a.ko.l;
        __builtin_nontemporal_store(x[j], (u32x4*)(dst + col0));
        __builtin_nontemporal_store(y[j], (u32x4*)(dst + col1));
      }
    }
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& r, hipStream_t st) {
  RotaryKernelArgs a;
  a.Q = (const __bf16*)r.Q; a.K = (const __bf16*)r.K; a.Qo = (__bf16*)r.Qo; a.Ko = (__bf16*)r.Ko;
  a.positions = r.positions;
  a.q = r.q; a.k = r.k; a.qo = r.qo; a.ko = r.ko;
  a.rows = (long long)r.B * r.L;
  a.Hq = r.Q ? r.Hq : 0;
  a.heads = a.Hq + (r.K ? r.Hkv : 0);
  a.L = r.L; a.units = r.d / 16; a.rot_units = r.rot / 16; a.half = r.rot / 2; a.start = r.start; a.gain = r.gain;
  a.by_L = FastDiv((uint32_t)r.L, (uint64_t)a.rows);
  for (int i = 0; i < kRotaryFreqs; ++i) a.turns[i] = r.turns[i];
  // As many tokens per workgroup as give every thread a unit.  More heads per thread spare sines and cosines, but what counts is to have
  // many loads in flight: 32768 tokens x 40 heads, d = 128, 16 tokens 139 us, 4: 123, 1: 124; 61 tokens x 40 heads, d = 64, 6.2, 5.5, 3.7.
  // (Ordinary instead of non-temporal loads and stores: 142 us with 16 tokens.)
  int tt_log2 = 0;
  while (tt_log2 < 4 && (a.heads * a.units << tt_log2) < 256) ++tt_log2;
  return launch_in_pieces((a.rows + (1 << tt_log2) - 1) >> tt_log2, [&](unsigned first, unsigned grid) {
    if (r.d == 128) {
      if (r.interleaved) rotary_kernel<true, 8><<<grid, 256, 0, st>>>(a, tt_log2, first);
      else rotary_kernel<false, 8><<<grid, 256, 0, st>>>(a, tt_log2, first);
    } else {
      if (r.interleaved) rotary_kernel<true, 4><<<grid, 256, 0, st>>>(a, tt_log2, first);
      else rotary_kernel<false, 4><<<grid, 256, 0, st>>>(a, tt_log2, first);
    }
  });
}

}  // namespace tsa
