// The paged cache: new rows of K and V into their pages (as they are, or in 8 bits), and sequences back as contiguous bf16.
// Movers: every row is read once and written once, HBM bounds them; short calls are a chain of look-ups (sequence, length,
// page) in front of one store.
//
// 8 bits.  A row x is kept as q = e4m3(x 2^-e), rounded to nearest even, with the smallest e for which max |x| <= 448 2^e (not below
// -126; 0 for a row of zeros).  A power of two costs no precision beside the rounding of the values themselves, and everything that
// is multiplied with it stays exact: x 2^-e here, q 2^e in bf16 on the way back, the scaling of scores and probabilities in the attention.
#include "cache_common.h"

namespace tsa {

using namespace cache_detail;

namespace {

struct WriteArgs {
  Batch b;
  const __bf16* K;
  const __bf16* V;
  char* kp;
  char* vp;
  uint8_t* ks;
  uint8_t* vs;
  long long k_t, k_h, v_t, v_h;  // element strides of a token and of a head
};

// Exponent byte of a row whose largest magnitude has these bf16 bits: 448 = 1.75 * 2^8, so e = exponent - 8, one more where the
// mantissa is above 1.75.  (A subnormal maximum lies far below 448 * 2^-126, the smallest range kept.)
__device__ __forceinline__ int exponent_byte(uint32_t bits) {
  if (bits == 0) return 127;
  const int byte = (int)(bits >> 7) - 8 + ((bits & 0x7f) > 0x60 ? 1 : 0);
  return max(byte, 1);                                   // (at most 248)
}

// A wavefront takes `TPW` consecutive tokens through a range of row groups: of a token's 2 Hkv rows (K's heads, then V's) d / 8 lanes hold
// one, 16 bytes each, 512 / d rows at a time.
template <int D, bool E4M3, int TPW>
__global__ __launch_bounds__(256) void cache_write_kernel(WriteArgs a, int groups, int groups_per_wave) {
  constexpr int LPR = D / 8, RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int t0 = (blockIdx.x * 4 + wave) * TPW;
  if (t0 >= a.b.n_tokens) return;
  const int g0 = blockIdx.y * groups_per_wave, g1 = min(groups, g0 + groups_per_wave);
  // where the tokens go: position, page (-1: nowhere)
  int seq = sequence_of(a.b, t0, lane), page[TPW], pos[TPW];
#pragma unroll
  for (int k = 0; k < TPW; ++k) {
    const int t = t0 + k;
    page[k] = -1;
    pos[k] = 0;
    if (t >= a.b.n_tokens) continue;
    while (seq < a.b.n_seqs && a.b.cu_q[seq + 1] <= t) ++seq;
    if (seq < 0 || seq >= a.b.n_seqs) continue;
    pos[k] = a.b.kv(seq) - (a.b.first(seq + 1) - t);
    if (pos[k] >= 0) page[k] = a.b.page(seq, pos[k]);
  }
  const int piece = lane % LPR;
  for (int grp = g0; grp < g1; ++grp) {
    const int r = grp * RPW + lane / LPR, Hkv = a.b.Hkv;
    const bool there = r < 2 * Hkv, is_v = r >= Hkv;
    const int h = is_v ? r - Hkv : r;
    const __bf16* src = (is_v ? a.V + h * a.v_h : a.K + h * a.k_h) + 8 * piece;
    const long long st = is_v ? a.v_t : a.k_t;
    u32x4 x[TPW];
#pragma unroll
    for (int k = 0; k < TPW; ++k)
      if (there && page[k] >= 0) x[k] = __builtin_nontemporal_load((const u32x4*)(src + (t0 + k) * st));
#pragma unroll
    for (int k = 0; k < TPW; ++k) {
      if (page[k] < 0) continue;                         // (the same in all lanes)
      const long long row = a.b.row(page[k], h, pos[k]);
      char* pool = is_v ? a.vp : a.kp;
      if (!E4M3) {
        if (there) *(u32x4*)(pool + row * (2 * D) + 16 * piece) = x[k];
        continue;
      }
      uint32_t big = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) big = max(big, max(x[k][i] & 0x7fffu, (x[k][i] >> 16) & 0x7fffu));
#pragma unroll
      for (int m = 1; m < LPR; m <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, m));
      const int byte = exponent_byte(big);
      const float s = exponent_value(254 - byte);        // 2^-e
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t p = x[k][2 * i], q = x[k][2 * i + 1];
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(p << 16) * s, __uint_as_float(p & 0xffff0000u) * s, 0, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(q << 16) * s, __uint_as_float(q & 0xffff0000u) * s, v, true);
        w[i] = (uint32_t)v;
      }
      if (there) {
        *(u32x2*)(pool + row * D + 8 * piece) = u32x2{w[0], w[1]};
        if (piece == 0) (is_v ? a.vs : a.ks)[row] = (uint8_t)byte;
      }
    }
  }
}

struct ReadArgs {
  Batch b;
  const char* kp;
  const char* vp;
  const uint8_t* ks;
  const uint8_t* vs;
  __bf16* K;
  __bf16* V;
  int L;
};

// A wavefront: 512 / d consecutive positions of one sequence and head, K and V, eight values per lane.  Rows behind the end of a sequence, and
// rows without a page, are zeros.  One row per lane: a look-up, a load and a store that depend on one another, hidden by many wavefronts
// (65536 tokens, 8 KV heads, d = 128, 8 bits: 75 us; two rows per lane 78, four 81, eight 98).
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadArgs a, int row_blocks, FastDiv by_blocks, FastDiv by_heads, unsigned first) {
  constexpr int LPR = D / 8, ROWS = 256 / LPR;             // lanes of a row, rows of a workgroup
  const uint32_t at = blockIdx.x + first, sh = by_blocks.div(at), block = at - sh * (uint32_t)row_blocks;
  const uint32_t seq = by_heads.div(sh), h = sh - seq * (uint32_t)a.b.Hkv;
  const int p = (int)block * ROWS + (int)threadIdx.x / LPR, piece = threadIdx.x % LPR;
  if (p >= a.L) return;
  const int id = p < a.b.kv((int)seq) ? a.b.page((int)seq, p) : -1;
  const long long row = a.b.row(max(id, 0), (int)h, p), out = (((long long)seq * a.b.Hkv + h) * a.L + p) * D + 8 * piece;
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (id >= 0) {
    if (E4M3) {
      const u32x2 kw = __builtin_nontemporal_load((const u32x2*)(a.kp + row * D + 8 * piece));
      const u32x2 vw = __builtin_nontemporal_load((const u32x2*)(a.vp + row * D + 8 * piece));
      const float ks = exponent_value(a.ks[row]), vs = exponent_value(a.vs[row]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x2 x = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kw[i >> 1], ks, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kw[i >> 1], ks, false);
        const bf16x2 y = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vw[i >> 1], vs, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vw[i >> 1], vs, false);
        k[i] = __builtin_bit_cast(uint32_t, x);
        v[i] = __builtin_bit_cast(uint32_t, y);
      }
    } else {
      k = __builtin_nontemporal_load((const u32x4*)(a.kp + row * (2 * D) + 16 * piece));
      v = __builtin_nontemporal_load((const u32x4*)(a.vp + row * (2 * D) + 16 * piece));
    }
  }
  __builtin_nontemporal_store(k, (u32x4*)(a.K + out));
  __builtin_nontemporal_store(v, (u32x4*)(a.V + out));
}

Batch batch_of(const CacheArgs& c) {
  Batch b;
  b.cu_q = c.cu_q; b.kv_len = c.kv_len; b.table = c.table;
  b.n_seqs = c.n_seqs; b.n_tokens = c.n_tokens; b.max_pages = c.max_pages; b.page_log2 = c.page_log2; b.n_pages = c.n_pages; b.Hkv = c.Hkv;
  return b;
}

template <int D, bool E4M3>
hipError_t launch_write(const WriteArgs& a, hipStream_t st) {
  constexpr int RPW = 512 / D;
  const int groups = (2 * a.b.Hkv + RPW - 1) / RPW;
  // Few tokens: a wavefront for every token and row group.  Many: two tokens per wavefront, whose look-ups and loads run together (43960 tokens, 8 KV
  // heads, d = 128, 8 bits: 53 us; four tokens 60, eight 63, one 56; ordinary loads of four 65).
  if (a.b.n_tokens <= 2048) {
    const dim3 grid((a.b.n_tokens + 3) / 4, groups);
    cache_write_kernel<D, E4M3, 1><<<grid, 256, 0, st>>>(a, groups, 1);
  } else {
    const dim3 grid((a.b.n_tokens + 7) / 8, 1);
    cache_write_kernel<D, E4M3, 2><<<grid, 256, 0, st>>>(a, groups, groups);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheArgs& c, const void* K, const void* V, hipStream_t st) {
  WriteArgs a;
  a.b = batch_of(c);
  a.K = (const __bf16*)K; a.V = (const __bf16*)V;
  a.kp = (char*)c.kp; a.vp = (char*)c.vp; a.ks = (uint8_t*)c.ks; a.vs = (uint8_t*)c.vs;
  a.k_t = c.k_t; a.k_h = c.k_h; a.v_t = c.v_t; a.v_h = c.v_h;
  if (c.d == 128) return c.e4m3 ? launch_write<128, true>(a, st) : launch_write<128, false>(a, st);
  return c.e4m3 ? launch_write<64, true>(a, st) : launch_write<64, false>(a, st);
}

hipError_t launch_cache_read(const CacheArgs& c, int L, void* K, void* V, hipStream_t st) {
  ReadArgs a;
  a.b = batch_of(c);
  a.kp = (const char*)c.kp; a.vp = (const char*)c.vp; a.ks = (const uint8_t*)c.ks; a.vs = (const uint8_t*)c.vs;
  a.K = (__bf16*)K; a.V = (__bf16*)V; a.L = L;
  const int rows = 2048 / c.d, blocks = (L + rows - 1) / rows;
  const long long all = (long long)c.n_seqs * c.Hkv * blocks;          // (checked to fit 31 bits by the caller)
  const FastDiv by_blocks(blocks, (uint64_t)all), by_heads(c.Hkv, (uint64_t)c.n_seqs * c.Hkv);
  return launch_in_pieces(all, [&](unsigned first, unsigned grid) {
    if (c.d == 128) {
      if (c.e4m3) cache_read_kernel<128, true><<<grid, 256, 0, st>>>(a, blocks, by_blocks, by_heads, first);
      else cache_read_kernel<128, false><<<grid, 256, 0, st>>>(a, blocks, by_blocks, by_heads, first);
    } else {
      if (c.e4m3) cache_read_kernel<64, true><<<grid, 256, 0, st>>>(a, blocks, by_blocks, by_heads, first);
      else cache_read_kernel<64, false><<<grid, 256, 0, st>>>(a, blocks, by_blocks, by_heads, first);
    }
  });
}

}  // namespace tsa
