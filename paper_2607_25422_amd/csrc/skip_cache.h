// The paged cache as its kernels see it (internal to libskip.so; the layout is in
// skip.h).
#pragma once

#include <cfloat>

#include "skip_common.h"
#include "skip_select.h"

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

// A batch's rows, tokens and prefixes.
struct CacheBatch {
  const int32_t *row_offsets, *lens, *prefix_ids, *prefix_lens;
  int B, H, G, heads_kv, total_rows, k_max, L_max;
};

// Items of sequences' own tokens are up to `cols` virtual rows over tiles of 32 tokens,
// those of prefixes up to kPrefixRows over tiles of kPrefixTile.
constexpr int kOwnTile = 32;
constexpr int kPrefixRows = 128, kPrefixTile = 64;

// Work is cut into equal runs of tiles, one a workgroup.  An item counts for a few
// tiles more than it has, which stand before its first: its queries, pages and first
// loads, and the join of its waves, take as long (short items one after the other in
// one workgroup: 512 items of 4 tiles on average 38 us without, 17 with).  A run that
// ends among them holds nothing of the item.
constexpr int kOwnStart = 8, kPrefixStart = 4;
// Tile of an item of nt at place u of its start + nt.
template <int START>
__device__ __forceinline__ int tile_at(int u, int nt) { return clampi(u - START, 0, nt); }

// 64 sequences, one a lane, and the tiles of their items.
struct SeqBlock {
  CacheSeq s;
  int P, first, run_rows;           // shared prefix; its run's first lane and rows
  int source;                       // the run's first lane with rows, whose pages are read
  int pre, own;                     // tiles (with their starts) of the prefix's items (of the run's first
                                    // lane) and of the sequence's own (TALL: of one key head)
  __device__ __forceinline__ static int row_tiles(const CacheBatch& a, int rows, int cols) {
    return (rows * a.G + cols - 1) / cols;
  }
  __device__ __forceinline__ static int own_tiles(int lo, int hi) {
    return max((hi + kOwnTile - 1) / kOwnTile - lo / kOwnTile, 1);
  }
  __device__ __forceinline__ static int prefix_tiles(int P) {
    return (P + kPrefixTile - 1) / kPrefixTile;
  }
  // tiles of kPrefixTile tokens that row tile i of a sequence's rows sees, at least one
  __device__ __forceinline__ static int tall_tiles(const CacheBatch& a, int n, int len, int i) {
    const int last = min((i + 1) * kPrefixRows, n * a.G) - 1;     // its last virtual row
    return max(prefix_tiles(len - n + last / a.G + 1), 1);
  }
  // tiles with their starts of the first `count` row tiles of a key head
  __device__ __forceinline__ static int tall_before(const CacheBatch& a, int n, int len,
                                                    int count) {
    int sum = 0;
    for (int i = 0; i < count; ++i) sum += tall_tiles(a, n, len, i) + kPrefixStart;
    return sum;
  }
  template <bool TALL>
  __device__ __forceinline__ void load(const CacheBatch& a, int b0, int cols) {
    const int lane = (int)__lane_id(), b = b0 + lane;
    s = CacheSeq{0, 0, 0};
    int id = -1, pl = 0;
    if (b < a.B) {
      s.load(a.row_offsets, a.lens, b, a.total_rows, a.k_max, a.L_max);
      if (a.prefix_ids) {
        id = a.prefix_ids[b];
        pl = a.prefix_lens[b];                         // (as it is: L_max makes no two alike)
        if (s.n > 0 && s.len < pl) id = -1;            // (does not hold the prefix)
      }
    }
    P = 0;
    first = lane;
    source = lane;
    run_rows = 0;
    pre = 0;
    if (a.prefix_ids) {
      const int id_b = __shfl_up(id, 1, kWave), pl_b = __shfl_up(pl, 1, kWave);
      const bool member = lane > 0 && id >= 0 && pl > 0 && id == id_b && pl == pl_b;
      const uint64_t starts = __ballot(!member);
      const uint64_t upto = lane == 63 ? ~0ull : (2ull << lane) - 1ull;
      first = 63 - __builtin_clzll(starts & upto);
      const uint64_t after = starts & ~upto;
      const int last = after ? __builtin_ctzll(after) - 1 : 63;    // of the run
      // (every lane takes part in the exchange)
      const int rows = __shfl(s.r0 + s.n, last, kWave) - __shfl(s.r0, first, kWave);
      // (a sequence that is passed over may have no pages left)
      source = __builtin_ctzll((__ballot(s.n > 0) & (~0ull << first)) | 1ull << 63);
      if (last > first) {
        P = pl;
        run_rows = rows;
        if (lane == first && run_rows > 0 && source <= last)     // (one holds all of it)
          pre = a.heads_kv * row_tiles(a, run_rows, kPrefixRows) *
                (prefix_tiles(P) + kPrefixStart);
      }
    }
    if (TALL) {
      own = s.n > 0 ? tall_before(a, s.n, s.len, row_tiles(a, s.n, kPrefixRows)) : 0;
      return;
    }
    own = s.n > 0 ? a.heads_kv * row_tiles(a, s.n, cols) *
                    (own_tiles(min(P, s.len), s.len) + kOwnStart) : 0;
  }
};

// The tiles of all items (of prefixes, or of sequences' own tokens) in order, and the
// sequence that a tile is of.
template <bool PREFIX, bool TALL = false>
struct SeqWalk {
  SeqBlock sb;                      // sequences sb0 ..
  int sb0, base, incl;              // tiles before them; running sums of theirs
  int cols;
  __device__ __forceinline__ int mine() const { return PREFIX ? sb.pre : sb.own; }
  __device__ __forceinline__ void block(const CacheBatch& a, int b0) {
    sb0 = b0;
    sb.load<TALL>(a, b0, cols);
    incl = (int)wave_incl_scan((uint32_t)mine());
  }
  __device__ __forceinline__ int block_tiles() const { return __builtin_amdgcn_readlane(incl, 63); }
  // All tiles; leaves the walk at the first sequences.
  template <class F>
  __device__ __forceinline__ int total(const CacheBatch& a, F&& each) {
    int W = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      block(a, b0);
      each(W);
      W += block_tiles();
    }
    base = 0;
    if (a.B > 64) block(a, 0);
    return W;
  }
  // The lane whose sequence tile u is of, and that sequence's first tile.
  __device__ __forceinline__ int seek(const CacheBatch& a, int u, int& start) {
    while (u >= base + block_tiles()) {
      base += block_tiles();
      block(a, sb0 + 64);
    }
    const int L = __popcll(__ballot(base + incl <= u));
    start = base + __builtin_amdgcn_readlane(incl - mine(), L);
    return L;
  }
  __device__ __forceinline__ int of_lane(int x, int L) const {
    return __builtin_amdgcn_readlane(x, L);
  }
};

// What the kernels of one call leave for the join, in the workspace: kCacheMeta ints
// a sequence, then the tiles of a run of own items, and of prefix items (or the tiles of
// a key head, where items go by key heads).
constexpr int kCacheMeta = 8;
struct CacheResults {
  int32_t* meta;
  float* part;                      // [2 runs][cols_own] parts of own items
  float* part_pre;                  // [2 runs][cols_pre] parts of prefix items
  float* whole;                     // [2][rows H] whole prefix items; whole own items
                                    // of sequences with a prefix
  int cols_own, cols_pre;
};
// Floats of a partial result of cols rows of D values: values, references, sums.
template <int D>
__device__ __host__ constexpr size_t part_floats(int cols) { return (size_t)cols * (D + 2); }
// Place of a whole result (D values, reference, sum).
template <int D>
__device__ __forceinline__ float* whole_at(const CacheResults& r, const CacheBatch& a, int own,
                                           size_t vr) {
  return r.whole + ((size_t)own * a.total_rows * a.H + vr) * (D + 4);
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

// The reference of weights 2^(logit - reference) once mx is the largest logit: 8 over it,
// so that it is rarely moved.  It stays finite: a logit past float32 then has an infinite
// weight, which makes its row NaN (an infinite reference would make all weights 0).
constexpr float kCacheOver = 8.f;
__device__ __forceinline__ float cache_reference(float mx) {
  return fminf(mx, FLT_MAX) + kCacheOver;
}
// A weight's exponent is s sc - reference in one multiply-add, whose product is exact, while
// the reference is a rounded one: half a step apart, which is 1 at 2^24 and past any
// exponent from 2^32 on.  Rows whose reference is farther than kCacheFar take their logits
// rounded as well, less the reference (over sc, so that the multiply-add serves both).
// (The branch is kept out of the loops' way: eight listed pages of one row 9.3 us, 9.1
// without it, 9.6 with its division before the loop; prompts the same, 1 % slower where a wave
// looks for such rows at every tile and not where references move.)
constexpr float kCacheFar = 16777216.f;
__device__ __forceinline__ float finite_reference(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ bool cache_far(float m) {
  return fabsf(finite_reference(m)) > kCacheFar;
}
// 1 / sc, where it is used (the compiler would put it before the loop).
__device__ __forceinline__ float far_back(float sc) {
  asm volatile("" : "+v"(sc));
  return 1.f / sc;
}
__device__ __forceinline__ float far_logit(float s, float sc, float ref, float back, bool far) {
  float z = s * sc;
  asm volatile("" : "+v"(z));                       // (not joined with the subtraction)
  return far ? (z - ref) * back : s;
}

CacheView cache_view(const skip_kv_cache_t& c);
inline CacheBatch cache_batch(const skip_problem_t& p, const skip_kv_cache_t& c,
                              const int32_t* row_offsets, const int32_t* lens,
                              const int32_t* prefix_ids, const int32_t* prefix_lens) {
  return CacheBatch{row_offsets, lens, prefix_ids, prefix_lens, p.B, p.H, p.H / c.heads_kv,
                    c.heads_kv, p.total_kept, p.k_max, p.L_max};
}
constexpr long long kMaxGrid = 1ll << 24;   // workgroups of up to 256 threads in a row
constexpr int kPrefixRuns = 512;            // workgroups of a call with shared prefixes

}  // namespace skip
