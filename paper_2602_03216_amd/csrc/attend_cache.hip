// Attention over the paged cache: the launches of a call, and the joining of parts.  Sequences with few rows: attend_cache_few.h, with many:
// attend_cache_many.hip.
#include "attend_cache_few.h"

namespace tsa {

using namespace cache_detail;
using namespace attend_cache_detail;

namespace {

template <int D, bool E4M3, int MB, bool ONCE>
__global__ __launch_bounds__(256, per_cu(D, E4M3, MB)) void attend_few_rows(Args a) {
  __shared__ __attribute__((aligned(1024))) char smem[Shape<D, E4M3, MB>::kLds];
  few_rows<D, E4M3, MB, ONCE, false>(a, smem, blockIdx.x);
}

template <int D, bool E4M3>
__global__ __launch_bounds__(512, 1) void attend_whole_tiles(Args a) {
  __shared__ __attribute__((aligned(1024))) char smem[Shape<D, E4M3, 1, 8>::kLds];
  few_rows<D, E4M3, 1, false, true>(a, smem, blockIdx.x);
}

constexpr int kMostParts = 1024;                         // shares, or parts of a row tile's keys: no row has more

// Row tiles that a share's end cuts: the shares that have a part of one deal its rows among them, four at a time.  (A workgroup for every share and group of
// four rows, most with nothing to do, is several rounds of the chip: 8 sequences x 4000 keys, 32 rows, 14.3 us, and 5.1 so.)  The first part is the second slot
// of its share, every later one the first slot of its share.  Wavefront r finds row r's largest max and its sum, then groups of lanes take every G-th
// part of all four.
template <int D>
__global__ __launch_bounds__(256) void join_few_rows(Args a) {
  constexpr int R = 4, LPR = D / 4, G = 256 / LPR, kBatch = 2;
  __shared__ float weight[R][kMostParts];
  __shared__ float meet[G][R][D];
  __shared__ float ml[R][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = tid / LPR, col = 4 * (tid % LPR);
  const Cut begins = a.cut[2 * blockIdx.x], ends = a.cut[2 * blockIdx.x + 1];
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {
    const Cut c = side ? ends : begins;
    if (c.parts <= 0) continue;
    const int share = max(0, (int)blockIdx.x - max(c.part, 0)), parts = min(c.parts, a.shares - share);
#pragma unroll 1
    for (int r0 = R * ((int)blockIdx.x - share + parts * blockIdx.y); r0 < c.rows; r0 += R * parts * gridDim.y) {
      const int rows = c.rows - r0;
      const long long first = (2LL * share + 1) * a.rt + r0, next = (2LL * share + 2) * a.rt + r0;
      const auto slot_of = [&](int w) -> long long { return w == 0 ? first : next + (long long)(w - 1) * 2 * a.rt; };
      f32x4 v[kBatch][R];
      const auto rows_from = [&](int w0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
          for (int r = 0; r < R; ++r)
            v[i][r] = w0 + i * G < parts && r < rows ? *(const f32x4*)(a.part_o + (slot_of(w0 + i * G) + r) * D + col) : f32x4{0, 0, 0, 0};
      };
      rows_from(grp);                                        // (the rows wait for nothing)
      float m = kNone, l = 0.f;
      if (wave < rows)
        for (int w = lane; w < parts; w += 64) {
          const long long slot = slot_of(w) + wave;
          const float mp = a.part_ml[2 * slot], lp = a.part_ml[2 * slot + 1], mn = fmaxf(m, mp);
          l = l * fast_exp2(m - mn) + lp * fast_exp2(mp - mn);
          m = mn;
          weight[wave][w] = mp;
        }
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) {
        const float mp = __shfl_xor(m, x), lp = __shfl_xor(l, x), mn = fmaxf(m, mp);
        l = l * fast_exp2(m - mn) + lp * fast_exp2(mp - mn);
        m = mn;
      }
      if (lane == 0) {
        ml[wave][0] = m;
        ml[wave][1] = l;
      }
      __syncthreads();
      f32x4 o[R];
#pragma unroll
      for (int r = 0; r < R; ++r) o[r] = f32x4{0, 0, 0, 0};
      for (int w0 = grp; w0 < parts; w0 += kBatch * G) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (w0 + i * G < parts && r < rows) o[r] += v[i][r] * fast_exp2(weight[r][w0 + i * G] - ml[r][0]);
        rows_from(w0 + kBatch * G);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) *(f32x4*)(&meet[grp][r][col]) = o[r];
      __syncthreads();
      for (int task = tid; task < R * D / 2; task += 256) {
        const int r = task / (D / 2), x = 2 * (task % (D / 2));
        if (r >= rows) continue;
        float v0 = 0.f, v1 = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          v0 += meet[g][r][x];
          v1 += meet[g][r][x + 1];
        }
        const int row = c.row0 + r0 + r, k = (int)a.by_g.div(row), tok = c.q0 + k, head = c.head * a.g + row - k * a.g;
        const float lt = ml[r][1], inv = lt > 0.f ? 1.0f / lt : 0.f;
        bf16x2 out;
        out[0] = (__bf16)(v0 * inv);
        out[1] = (__bf16)(v1 * inv);
        *(bf16x2*)(a.O + tok * a.o_t + head * a.o_h + x) = out;
        if (a.lse && x == 0) a.lse[(long long)tok * a.Hq + head] = lt == 0.f ? -INFINITY : (ml[r][0] + log2f(lt)) * kLn2;
      }
      __syncthreads();
    }
  }
}

// Rows whose keys are cut into parts (many rows): a workgroup takes 16 rows of a row tile, D / 4 lanes a row, which they sum part by part.
template <int D>
__global__ __launch_bounds__(256) void join_many_rows(Args a) {
  constexpr int LPR = D / 4, G = 256 / LPR, kRows = 16, kBatch = 8;
  const int lane = threadIdx.x & 63, grp = threadIdx.x / LPR, col = 4 * (threadIdx.x % LPR);
  const int slot = blockIdx.x, h = blockIdx.y;
  const int seq = last_up_to(a.b.n_seqs, slot, lane, [&](int i) { return first_slot(a, i); });
  if (seq < 0 || seq >= a.b.n_seqs) return;
  const ManyTile x = many_tile(a, seq, slot - first_slot(a, seq));
  if (!x.there || x.parts == 1) return;
#pragma unroll
  for (int k = 0; k < kRows; k += G) {
    const int in_tile = kRows * blockIdx.z + k + grp, row = x.row0 + in_tile;
    if (row >= x.rows) continue;
    const long long first = ((long long)slot * a.b.Hkv + h) * a.splits * kManyRows + in_tile;
    f32x4 o = {0, 0, 0, 0};
    float m = kNone, l = 0.f;
    for (int w0 = 0; w0 < x.parts; w0 += kBatch) {
      f32x4 v[kBatch];
      float mp[kBatch], lp[kBatch], mn = m;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const long long at = first + (long long)min(w0 + i, x.parts - 1) * kManyRows;
        mp[i] = a.many_ml[2 * at];
        lp[i] = a.many_ml[2 * at + 1];
        v[i] = *(const f32x4*)(a.many_o + at * D + col);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) mn = fmaxf(mn, mp[i]);
      const float alpha = fast_exp2(m - mn);
      m = mn;
      l *= alpha;
      o *= alpha;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const float w = w0 + i < x.parts ? fast_exp2(mp[i] - mn) : 0.f;
        l += lp[i] * w;
        o += v[i] * w;
      }
    }
    const int k_tok = (int)a.by_g.div(row), tok = x.q0 + k_tok, head = h * a.g + row - k_tok * a.g;
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    bf16x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = (__bf16)(o[i] * inv);
    *(bf16x4*)(a.O + tok * a.o_t + head * a.o_h + col) = out;
    if (a.lse && col == 0) a.lse[(long long)tok * a.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// How a call is cut, from what the host knows: whether any sequence may have many rows, rows of a tile and shares of the ones that have few,
// and for many the slots for row tiles and the parts that their keys are cut into.
struct Plan {
  bool few, many, fits, once, whole, by_rows;
  int mb, tiles, rows, shares, slots, splits, short_splits, long_keys;      // rows: of a tile, as many as there will be
};
Plan plan_of(const CacheArgs& c) {
  const int g = c.Hq / c.Hkv, most = c.max_q > 0 && c.max_q < c.n_tokens ? c.max_q : c.n_tokens;
  Plan p;
  const long long cap = (long long)c.max_pages << c.page_log2, seen = c.window && c.window + (long long)most < cap ? c.window + (long long)most : cap;
  // (steps are counted in 32 bits on the device)
  const auto steps = [&](long long rows) { return (double)c.Hkv * (rows / 16 + c.n_seqs) * ((cap + kStep - 1) / kStep + 2048); };
  const long long rows_all = (long long)c.n_tokens * g, rows_few = rows_all < (long long)c.n_seqs * kFewRows ? rows_all : (long long)c.n_seqs * kFewRows;
  p.many = (long long)most * g > kFewRows || steps(rows_all) >= 4.0e9;
  p.few = !p.many || c.n_seqs > 1;
  p.fits = !p.few || steps(p.many ? rows_few : rows_all) < 4.0e9;
  const int rows = p.many ? g : most * g;                // (beside prompts: single tokens, most likely)
  // Rows of a tile.  Larger tiles read K and V fewer times, smaller ones start and end sooner and are more of them.  28 / 4 heads, us with tiles of
  // 16 / 32 / 64 rows: 32 sequences x 8000 keys, 3 new tokens (21 rows) bf16 156 / 96 / 99, 8 bits 87 / 58 / 90; 8 new tokens (56 rows) 292 / 163 / 103 and
  // 153 / 94 / 94 (d = 64: 149 / 87 / 59 and 91 / 64 / 53); 200 x 500, 56 rows, 139 / 92 / 87 and 87 / 69 / 80; 2 x 300, 56 rows, 11.6 / 15.0 / 18.1 and
  // 11.0 / 13.9 / 17.3; 1 x 2000 12.6 / 14.0 / 17.5.  So 16 rows where the steps of the whole capacity run at once whatever the lengths are.
  const bool small = (long long)c.n_seqs * c.Hkv * ((seen + kStep - 1) / kStep) <= 512;
  p.mb = rows <= 16 || small ? 1 : rows <= 32 || (c.e4m3 && c.d == 128) ? 2 : 4;
  // K and V that no other tile reads again pass the caches by: 64 sequences x 8192 keys, 8 KV heads, us without / with: bf16 363 / 329, 8 bits 198 / 183,
  // d = 64 186 / 169 and 106 / 95; short ones lose little (1 x 2000 11.3 / 11.7).  Where several tiles read them it costs: four drafted tokens of 7 heads
  // a group over 1 x 2000, 23.5 / 25.9.
  p.once = rows <= 16 * p.mb;
  p.rows = !p.many && most * g < 16 * p.mb ? most * g : 16 * p.mb;
  // Short contexts of few sequences: whole row tiles by workgroups of twice the wavefronts, at most one per CU, without parts and so without a second
  // launch (3 us of the host's time beside what follows).  us in shares / whole, 8 KV heads, one token: 1 sequence x 500 keys bf16 10.8 / 9.3, 8 bits 10.3 /
  // 7.8, d = 64 9.6 / 6.0 and 9.5 / 5.7; x 1000 11.2 / 13.9, 10.8 / 11.7, 9.8 / 9.0, 9.6 / 7.6; 32 sequences x 1000 30.4 / 26.7, 22.5 / 17.6, 20.2 / 15.8,
  // 17.4 / 12.2; x 2000 49.7 / 48.8, 32.6 / 29.3, 29.8 / 26.5, 22.9 / 18.5; 64 x 1000 48.0 / 51.3, 31.2 / 34.2, 27.7 / 29.6, 22.8 / 22.1.  Few tiles wait for every
  // step's latency, so many keys are better dealt out; rows of 128 bytes or less, or 128 tiles and more, bear twice as many.
  p.tiles = (most * g + 15) / 16;
  const long long whole_tiles = (long long)c.n_seqs * c.Hkv * p.tiles;
  p.whole = !p.many && p.mb == 1 && whole_tiles <= 256 && seen <= (512 << ((c.d == 64 || c.e4m3) + (whole_tiles >= 128)));
  p.shares = p.whole ? 1 : 256 * per_cu(c.d, c.e4m3, p.mb);
  // slots for row tiles, the fewer of two kinds (first_slot)
  const long long by_seq = rows_all / kManyRows + c.n_seqs, by_rows = 2 * rows_all / (kManyRows + 1);
  p.by_rows = p.few && by_rows < by_seq;
  p.slots = (int)(p.by_rows ? by_rows : by_seq);
  // Row tiles, as if sequences of the most tokens made up the rows; parts as many as run at once with them (two workgroups a CU, of d = 64 in bf16 three).  One part more, so that no
  // place stays empty, starts a second round: 32 / 8 heads, bf16, us with the last part that fits / one more: 300 tokens over 6000 keys 51 / 61, 700 over
  // 16384 213 / 269, 4 x 300 over 6000 150 / 168, with a window of 1024 40 / 60; twice the parts: 63, 211, 166, 61.
  const auto tiles_of = [&](long long tokens) { return (tokens * g + kManyRows - 1) / kManyRows; };
  const long long full = most > 0 ? c.n_tokens / most : 0;
  const long long tiles = c.Hkv * (full > 0 && full <= c.n_seqs ? full * tiles_of(most) + tiles_of(c.n_tokens - full * most) : tiles_of(c.n_tokens));
  const long long most_parts = cap / (kTile * kPartTiles);
  const long long places = c.d == 64 && !c.e4m3 ? 768 : 512;
  const auto parts = [&](long long s) { return s > most_parts ? most_parts : s; };
  const auto bounded = [](long long s) { return (int)(s < 1 ? 1 : s > kMostParts ? kMostParts : s); };
  const long long s = places / (tiles > 0 ? tiles : 1);
  p.splits = p.short_splits = bounded(parts(s));
  p.long_keys = 0;
  // Over long contexts more than that; how long they are, the device knows (the table may be a model's longest: 2176 tokens over 2500 keys, 32 / 8 heads, bf16,
  // with a table of 131072 positions 94 us in the parts of a long context, 66 in those of a short one).
  const auto over = [&](long long keys, long long more) {
    if (seen < keys) return;
    p.long_keys = (int)keys;
    p.splits = bounded(parts(more));
  };
  // Where one round leaves a quarter of the places empty: parts that fill two rounds, as long as they are long (28 / 4 heads, 1500 tokens, one part / three:
  // over 16384 keys bf16 369 / 338, d = 64 in 8 bits 280 / 219; over 6000 137 / 136, 103 / 90; over 2500 58 / 71, 47 / 51).
  const long long two = tiles > 0 ? 2 * places / tiles : 0;
  if (4 * tiles * s < 3 * places && 4 * tiles * two >= 7 * places) over(1536 * two, two);
  // ... and three parts where the tiles are a few more than the places (32 / 8 heads, 2176 tokens, bf16, one part / three: over 16384 keys 693 / 576, over 6000
  // 215 / 218).
  if (tiles > places && 3 * tiles <= 4 * places) over(8192, 3);
  return p;
}

struct Workspace {
  size_t part_ml, part_o, many_ml, many_o, total;
};
Workspace workspace_of(const CacheArgs& c, const Plan& p) {
  Workspace w;
  size_t at = align256(2 * (size_t)p.shares * sizeof(Cut));
  auto take = [&](size_t n) { const size_t x = at; at += align256(n); return x; };
  const size_t few = 2 * (size_t)p.shares * 16 * p.mb, many = p.many && p.splits > 1 ? (size_t)p.slots * c.Hkv * p.splits * kManyRows : 0;
  w.part_ml = take(few * 2 * 4);
  w.part_o = take(few * c.d * 4);
  w.many_ml = take(many * 2 * 4);
  w.many_o = take(many * c.d * 4);
  w.total = at;
  return w;
}

template <int D, bool E4M3>
hipError_t launch(Args& a, const Plan& p, hipStream_t st) {
  hipError_t e;
  a.few = p.many ? (p.few ? kFewRows : 0) : 0x7fffffff;
  // with tiles of 16 rows the shares run in the same launch as the rows of many, behind them: in its tail
  const bool both = p.many && p.few && p.mb == 1;
  if (p.many && (e = launch_attend_many(a, D, E4M3, both ? p.shares : 0, st)) != hipSuccess) return e;
  if (p.whole) {
    attend_whole_tiles<D, E4M3><<<a.b.n_seqs * p.tiles * a.b.Hkv, 512, 0, st>>>(a);
    return hipGetLastError();
  }
  if (p.few && !both) {
    if (p.mb == 4) {
      if constexpr (!(E4M3 && D == 128)) attend_few_rows<D, E4M3, 4, true><<<p.shares, 256, 0, st>>>(a);
      else return hipErrorInvalidConfiguration;            // (those have tiles of at most 32 rows)
    } else if (p.mb == 2) {
      bool once = true;
      if constexpr (E4M3 && D == 128) once = p.once;     // (the only ones whose 33 to 64 rows are not one tile)
      if (once) attend_few_rows<D, E4M3, 2, true><<<p.shares, 256, 0, st>>>(a);
      else if constexpr (E4M3 && D == 128) attend_few_rows<D, E4M3, 2, false><<<p.shares, 256, 0, st>>>(a);
    } else if (p.once) attend_few_rows<D, E4M3, 1, true><<<p.shares, 256, 0, st>>>(a);
    else attend_few_rows<D, E4M3, 1, false><<<p.shares, 256, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (p.few) {
    const int groups = (p.rows + 3) / 4, at_once = 1024 / p.shares;
    join_few_rows<D><<<dim3(p.shares, groups < at_once ? groups : at_once), 256, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (p.many && p.splits > 1) {
    join_many_rows<D><<<dim3(a.slots, a.b.Hkv, kManyRows / 16), 256, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t attend_cache_ws_bytes(const CacheArgs& c) {
  const Plan p = plan_of(c);
  return p.fits ? workspace_of(c, p).total : 0;
}

hipError_t launch_attend_cache(const CacheArgs& c, const void* Q, void* O, float* lse, void* ws, hipStream_t st) {
  Args a;
  a.b.cu_q = c.cu_q; a.b.kv_len = c.kv_len; a.b.table = c.table;
  a.b.n_seqs = c.n_seqs; a.b.n_tokens = c.n_tokens; a.b.max_pages = c.max_pages; a.b.page_log2 = c.page_log2; a.b.n_pages = c.n_pages; a.b.Hkv = c.Hkv;
  a.Q = (const __bf16*)Q; a.kp = (const char*)c.kp; a.vp = (const char*)c.vp; a.ks = (const uint8_t*)c.ks; a.vs = (const uint8_t*)c.vs;
  a.O = (__bf16*)O; a.lse = lse;
  a.q_t = c.q_t; a.q_h = c.q_h; a.o_t = c.o_t; a.o_h = c.o_h;
  a.Hq = c.Hq; a.g = c.Hq / c.Hkv; a.window = c.window; a.c = c.scale * kLog2e;
  a.by_g = FastDiv((uint32_t)a.g, (uint64_t)c.n_tokens * a.g + 1);
  const Plan p = plan_of(c);
  const Workspace w = workspace_of(c, p);
  char* base = (char*)ws;
  a.cut = (Cut*)base;
  a.part_ml = (float*)(base + w.part_ml);
  a.part_o = (float*)(base + w.part_o);
  a.many_ml = (float*)(base + w.many_ml);
  a.many_o = (float*)(base + w.many_o);
  a.rt = 16 * p.mb; a.shares = p.shares; a.whole = p.tiles; a.slots = p.slots; a.by_rows = p.by_rows;
  a.splits = p.splits; a.short_splits = p.short_splits; a.long_keys = p.long_keys;
  if (c.d == 128) return c.e4m3 ? launch<128, true>(a, p, st) : launch<128, false>(a, p, st);
  return c.e4m3 ? launch<64, true>(a, p, st) : launch<64, false>(a, p, st);
}

}  // namespace tsa
