// The paged cache as its kernels see it (internal to libskip.so; the layout is in
// skip.h).
#pragma once

#include "skip_common.h"

namespace skip {

struct CacheView {
  bf16_t* k;                     // [n_pages][heads_kv][page][d_h]
  bf16_t* v;
  bf16_t* mean;                  // [n_pages][heads_kv][d_h], or NULL
  const int32_t* table;          // [B][pages_max]
  long long n_pages;
  int heads_kv, pages_max, shift;   // a page holds 1 << shift tokens
  // the physical page of a sequence's page j, or -1 where there is none
  __device__ __forceinline__ int page(int b, int j) const {
    if (j < 0 || j >= pages_max) return -1;
    const int at = table[(size_t)b * pages_max + j];
    return at >= 0 && (long long)at < n_pages ? at : -1;
  }
  // elements before a physical page of one key head
  template <int D>
  __device__ __forceinline__ size_t base(int at, int hk) const {
    return ((size_t)(uint32_t)at * heads_kv + hk) * ((size_t)D << shift);
  }
};

// The rows and tokens of a sequence: rows r0 .. r0 + n - 1, the last n of len
// tokens.
struct CacheSeq {
  int r0, n, len;
  __device__ __forceinline__ void load(const int32_t* row_offsets, const int32_t* lens, int b,
                                       int total_rows, int k_max, int L_max) {
    int r1;
    range_of(row_offsets, b, total_rows, r0, r1);
    n = min(r1 - r0, k_max);
    len = clampi(lens[b], 0, L_max);
  }
};

// All ones in the halves of a word that hold a bf16 infinity or NaN.
__device__ __forceinline__ uint32_t bf16_odd_pair(uint32_t x) {
  return ((x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) |
         ((x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// The sequence of a row (every lane the same), or -1: a row behind the last one, or
// one that a sequence has no place for.
__device__ __forceinline__ int seq_of_row(const int32_t* row_offsets, const int32_t* lens, int B,
                                          int total_rows, int k_max, int L_max, int row,
                                          CacheSeq& s) {
  const int lane = (int)__lane_id();
  int b = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const bool behind = b0 + lane < B && clampi(row_offsets[b0 + lane + 1], 0, total_rows) <= row;
    const int n = __popcll(__ballot(behind));
    b += n;
    if (n < 64) break;
  }
  if (b >= B) return -1;
  s.load(row_offsets, lens, b, total_rows, k_max, L_max);
  return row >= s.r0 && row < s.r0 + s.n ? b : -1;
}

// Value of lane l ^ 16 and l ^ 32 joined with the lane's own by op, in every lane.
template <class F>
__device__ __forceinline__ float over_groups(float x, F op) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t w = __float_as_uint(op(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

CacheView cache_view(const skip_kv_cache_t& c);

}  // namespace skip
