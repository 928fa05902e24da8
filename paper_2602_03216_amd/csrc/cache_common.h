// Pieces shared by the kernels of the paged cache (cache.hip: rows into it and out of it; attend_cache.hip: attention over it).
//
// The pool of K, and that of V, is [n_pages][Hkv][page_size][d]: one head's keys of a page are one contiguous piece.  Elements are
// bf16, or e4m3 (4 exponent bits, 3 mantissa bits, largest finite value 448) with one byte per row in [n_pages][Hkv][page_size]: the
// exponent e + 127 of the power of two that the row's values are multiplied by.
// Device-side counts and tables are not trusted with addresses: whatever they hold, every access stays inside the caller's tensors.
#pragma once

#include "tsa_internal.h"

namespace tsa {

namespace cache_detail {

struct Batch {
  const int32_t* cu_q;           // [n_seqs + 1]; NULL: no new tokens (reading back)
  const int32_t* kv_len;         // [n_seqs]
  const int32_t* table;          // [n_seqs][max_pages]
  int n_seqs, n_tokens, max_pages, page_log2, n_pages, Hkv;

  __device__ __forceinline__ int kv(int i) const { return min(max(kv_len[i], 0), max_pages << page_log2); }
  // first token at or behind sequence i's place in the packed rows, never outside [0, n_tokens]
  __device__ __forceinline__ int first(int i) const { return min(max(cu_q[i], 0), n_tokens); }
  // page of position p of sequence i (p inside the table), -1: none
  __device__ __forceinline__ int page(int i, int p) const {
    const int id = table[(long long)i * max_pages + (p >> page_log2)];
    return (unsigned)id < (unsigned)n_pages ? id : -1;
  }
  // row of the pools (of d elements; also the place of the scale) of head h, position p on page id
  __device__ __forceinline__ long long row(int id, int h, int p) const {
    return (((long long)id * Hkv + h) << page_log2) + (p & ((1 << page_log2) - 1));
  }
};

// The last i in 0 .. n_seqs with key(i) <= t, by the whole wavefront together, 64 samples of the ascending keys per round (one round up to
// 64 sequences, two up to 4096); -1: none.  t is the same in all lanes.
template <typename F>
__device__ __forceinline__ int last_up_to(int n_seqs, int t, int lane, F&& key) {
  int lo = 0, n = n_seqs + 1;                            // candidates lo .. lo + n - 1
  while (n > 0) {
    const int stride = (n + 63) >> 6, i = lo + lane * stride;
    const bool up_to = lane * stride < n && key(i) <= t;
    const int k = __popcll(__builtin_amdgcn_ballot_w64(up_to));              // ascending: lanes 0 .. k - 1
    if (k == 0) break;
    lo += (k - 1) * stride + 1;
    n = min(stride - 1, n_seqs + 1 - lo);
  }
  return lo - 1;
}
// Sequence that token t of the packed rows belongs to: n_seqs for a token behind the last sequence, -1 for one in front of the first.
__device__ __forceinline__ int sequence_of(const Batch& b, int t, int lane) {
  return last_up_to(b.n_seqs, t, lane, [&](int i) { return b.cu_q[i]; });
}

__device__ __forceinline__ float exponent_value(uint32_t byte) { return __uint_as_float(byte << 23); }     // 2^(byte - 127), byte 1 .. 254

}  // namespace cache_detail

}  // namespace tsa
