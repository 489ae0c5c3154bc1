// A paged cache of keys and values: new tokens rotated by their positions and
// appended, and the pages that a score selects for each of them.
#include <algorithm>

#include "skip_cache.h"
#include "skip_common.h"
#include "skip_internal.h"
#include "skip_select.h"

namespace skip {

// ---------------------------------------------------------------------------
// Append.  For the new token at position t (or the position given for it),
//   a_i = t f_i,  (x, y) -> (x cos a_i - y sin a_i, y cos a_i + x sin a_i)
// on the feature pairs i of every query and key head, one rounding to bf16; keys and
// values into the token's page; the mean of the page's keys up to the sequence's
// last token.
//
// A workgroup takes one page that new tokens go to, of one key head: its keys,
// values and the group's queries of those tokens, and the page's mean, for which it
// reads the keys that were there (so that the mean is the keys', whatever was
// appended, cut off or written again before).  Memory bounds it: a new token's rows
// are read once and written once (16 prompts of 230 to 544 tokens, 32 heads of 128 over
// 8: 43 us for 168 MB, 3.9 TB/s where a copy reaches 6.2; the angles, which stand before the
// first loads, are made again by each key head's workgroup).
constexpr int kAppThreads = 256;
constexpr int kAppTokens = 32;             // tokens whose angles are in LDS at a time
constexpr int kAppMaxHalf = 64;            // rotated pairs of a row

struct AppendArgs {
  CacheView cache;
  const void *q, *k, *v;
  long long qs, ks, vs;                    // elements from one row to the next
  const float* freq;
  const int32_t *row_offsets, *lens, *positions;
  bf16_t* q_out;
  int B, H, G, total_rows, k_max, L_max, half, pairs;
};

__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  return u32x4{pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]), pack2_bf16(x[4], x[5]),
               pack2_bf16(x[6], x[7])};
}

// Features 8 c .. + 7 of a row, and those that rotation joins them with.
template <typename T>
struct Chunk {
  typedef typename std::conditional<sizeof(T) == 2, u32x4, float4>::type Half;
  static constexpr int N = sizeof(T) / 2;          // 16-byte words of eight elements
  Half x[N], y[N];
  __device__ __forceinline__ void load(const T* row, int c, int half, int pairs) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = reinterpret_cast<const Half*>(row + 8 * c)[i];
    if (!pairs && 8 * c < 2 * half) {
      const T* other = row + (8 * c < half ? 8 * c + half : 8 * c - half);
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = reinterpret_cast<const Half*>(other)[i];
    }
  }
  static __device__ __forceinline__ void floats(const Half (&h)[N], float (&f)[8]) {
    if constexpr (N == 1) {
      unpack8_bf16(h[0], f);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[4 * i] = h[i].x, f[4 * i + 1] = h[i].y;
        f[4 * i + 2] = h[i].z, f[4 * i + 3] = h[i].w;
      }
    }
  }
  // rotated by the angles of its token (cosine and sine of pair i at cs[i])
  __device__ __forceinline__ u32x4 rotated(int c, int half, int pairs, const float2* cs) const {
    float a[8];
    floats(x, a);
    if (8 * c < 2 * half) {
      if (pairs) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 w = cs[4 * c + e];
          const float p = a[2 * e], q = a[2 * e + 1];
          a[2 * e] = p * w.x - q * w.y;
          a[2 * e + 1] = q * w.x + p * w.y;
        }
      } else {
        float b[8];
        floats(y, b);
        const bool low = 8 * c < half;
        const float2* w = cs + (low ? 8 * c : 8 * c - half);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = a[e] * w[e].x + (low ? -b[e] : b[e]) * w[e].y;
      }
    }
    return pack8(a);
  }
  __device__ __forceinline__ u32x4 rounded() const {
    float a[8];
    floats(x, a);
    return pack8(a);
  }
};

// A page that new tokens go to: tokens t0 .. end - 1 of it are held, from `first` on new.
struct AppendPage {
  int t0, first, end, row0;                        // row0: the row of token 0
  int at;                                          // the physical page, or -1
  // The slot-th such page of the batch (every wave the same): prefix sums of the pages
  // that each sequence's new tokens go to.
  __device__ __forceinline__ bool find(const AppendArgs& a, int slot) {
    const int lane = threadIdx.x & 63, shift = a.cache.shift;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      int pages = 0;
      CacheSeq s{0, 0, 0};
      if (b0 + lane < a.B) {
        s.load(a.row_offsets, a.lens, b0 + lane, a.total_rows, a.k_max, a.L_max);
        if (s.n > 0 && s.len > 0)
          pages = ((s.len - 1) >> shift) - (max(s.len - s.n, 0) >> shift) + 1;
      }
      const int incl = (int)wave_incl_scan((uint32_t)pages);
      const int total = __builtin_amdgcn_readlane(incl, 63);
      if (slot < total) {
        const int l = __popcll(__ballot(incl <= slot));
        const int r0 = __builtin_amdgcn_readlane(s.r0, l), n = __builtin_amdgcn_readlane(s.n, l);
        const int len = __builtin_amdgcn_readlane(s.len, l);
        const int pg = (max(len - n, 0) >> shift) + slot -
                       __builtin_amdgcn_readlane(incl - pages, l);
        t0 = pg << shift;
        first = max(len - n, t0);
        end = min(len, t0 + (1 << shift));
        row0 = r0 + n - len;
        at = a.cache.page(b0 + l, pg);
        return true;
      }
      slot -= total;
    }
    return false;
  }
};

// The mean of a page's keys from the sums that TL threads a chunk hold.
template <int D, int TL>
__device__ __forceinline__ void store_mean(const AppendArgs& a, const AppendPage& p, int hk,
                                           const float (&sum)[8], float (*sums)[D]) {
  const int tid = threadIdx.x, c = tid % (D / 8), tl = tid / (D / 8);
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[tl][8 * c + e] = sum[e];
  __syncthreads();
  if (tid >= D / 2) return;
  float x = 0.f, y = 0.f;
  for (int i = 0; i < TL; ++i) {
    x += sums[i][2 * tid];
    y += sums[i][2 * tid + 1];
  }
  const float inv = 1.f / (float)(p.end - p.t0);
  reinterpret_cast<uint32_t*>(a.cache.mean + ((size_t)(uint32_t)p.at * a.cache.heads_kv + hk) *
                                                 D)[tid] = pack2_bf16(x * inv, y * inv);
}
// Sums of the keys of tokens t0 .. t1 - 1 as the page holds them.
template <int D, int TL>
__device__ __forceinline__ void sum_keys(const bf16_t* kp, int t0, int t1, float (&sum)[8]) {
  const int c = threadIdx.x % (D / 8), tl = threadIdx.x / (D / 8);
#pragma unroll 4
  for (int t = t0 + tl; t < t1; t += TL) {
    float x[8];
    unpack8_bf16(*reinterpret_cast<const u32x4*>(kp + (size_t)(t - t0) * D + 8 * c), x);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += x[e];
  }
}

// PIECES: a workgroup takes 32 tokens of the page and four of the group's queries, and
// the mean is left to a launch of its own.
constexpr int kAppHeads = 4;
template <typename T, int D, bool PIECES>
__global__ void __launch_bounds__(kAppThreads)
cache_append_kernel(AppendArgs a) {
  constexpr int C = D / 8;                         // 16-byte chunks of a row
  constexpr int TL = kAppThreads / C;              // tokens side by side
  __shared__ float2 cs[kAppTokens][kAppMaxHalf];
  __shared__ float sums[PIECES ? 1 : TL][D];
  const int tid = threadIdx.x, hk = blockIdx.y, shift = a.cache.shift;
  AppendPage p;
  const int pieces = PIECES ? 1 << (shift - 5) : 1;
  if (!p.find(a, blockIdx.x / pieces)) return;
  const int t0 = p.t0, row0 = p.row0, at = p.at;
  int first = p.first, end = p.end;
  if (PIECES) {
    const int u = t0 + kAppTokens * (blockIdx.x % pieces);
    first = max(first, u);
    end = min(end, u + kAppTokens);
    if (first >= end) return;
  }
  const size_t base = a.cache.base<D>(max(at, 0), hk);
  bf16_t* const kp = a.cache.k + base;
  bf16_t* const vp = a.cache.v + base;
  const int c = tid % C, tl = tid / C;

  // keys that were there
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (!PIECES && a.cache.mean && at >= 0) sum_keys<D, TL>(kp, t0, first, sum);

  for (int u = max(first, 0); u < end; u += kAppTokens) {
    const int nt = min(end - u, kAppTokens);
    for (int i = tid; i < nt * a.half; i += kAppThreads) {
      const int j = i / a.half, f = i - j * a.half;
      const int pos = a.positions ? a.positions[row0 + u + j] : u + j;
      // the angle in revolutions, reduced in 64 bits: an angle of a far position has
      // no bits left in 32
      const double rev = (double)pos * (double)a.freq[f] * 0.15915494309189533577;
      const float frac = (float)(rev - rint(rev));
      cs[j][f] = make_float2(cospif(2.f * frac), sinpif(2.f * frac));
    }
    __syncthreads();
    // a token's key and value; then the group's queries, four rows of loads in flight
    for (int j = PIECES && blockIdx.z > 0 ? nt : tl; j < nt; j += TL) {
      const int t = u + j;
      const size_t r = (size_t)(row0 + t);
      Chunk<T> kx, vx;
      kx.load(static_cast<const T*>(a.k) + r * a.ks + (size_t)hk * D, c, a.half, a.pairs);
      vx.load(static_cast<const T*>(a.v) + r * a.vs + (size_t)hk * D, c, 0, 0);
      const u32x4 ko = kx.rotated(c, a.half, a.pairs, cs[j]);
      if (at >= 0) {
        *reinterpret_cast<u32x4*>(kp + (size_t)(t - t0) * D + 8 * c) = ko;
        *reinterpret_cast<u32x4*>(vp + (size_t)(t - t0) * D + 8 * c) = vx.rounded();
      }
      float x[8];
      unpack8_bf16(ko, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += x[e];
    }
    if (a.q) {
      constexpr int U = 4;
      const int h0 = PIECES ? kAppHeads * blockIdx.z : 0;
      const int heads = PIECES ? min(a.G - h0, kAppHeads) : a.G, n = nt * heads;
      for (int i = tl; i < n; i += U * TL) {
        Chunk<T> x[U];
        int tok[U], h[U];
#pragma unroll
        for (int m = 0; m < U; ++m) {
          const int k = min(i + m * TL, n - 1);
          tok[m] = k / heads;
          h[m] = hk * a.G + h0 + (k - tok[m] * heads);
          x[m].load(static_cast<const T*>(a.q) + (size_t)(row0 + u + tok[m]) * a.qs +
                        (size_t)h[m] * D, c, a.half, a.pairs);
        }
#pragma unroll
        for (int m = 0; m < U; ++m)
          if (i + m * TL < n)
            *reinterpret_cast<u32x4*>(a.q_out + ((size_t)(row0 + u + tok[m]) * a.H + h[m]) * D +
                                      8 * c) = x[m].rotated(c, a.half, a.pairs, cs[tok[m]]);
      }
    }
    __syncthreads();
  }
  if constexpr (!PIECES)
    if (a.cache.mean && at >= 0) store_mean<D, TL>(a, p, hk, sum, sums);
}

template <int D>
__global__ void __launch_bounds__(kAppThreads)
cache_mean_kernel(AppendArgs a) {
  constexpr int TL = kAppThreads / (D / 8);
  __shared__ float sums[TL][D];
  AppendPage p;
  if (!p.find(a, blockIdx.x) || p.at < 0) return;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  sum_keys<D, TL>(a.cache.k + a.cache.base<D>(p.at, blockIdx.y), p.t0, p.end, sum);
  store_mean<D, TL>(a, p, blockIdx.y, sum, sums);
}

// ---------------------------------------------------------------------------
// Selection.  For the new token at position t and key head h,
//   s_j = sum over features of (sum over the head's group of q) * mean key of page j
// for the pages j <= t / page, and the n_sel pages of the largest s_j (ties: the
// lower page), the n_first first and n_last last among them whatever their scores.
// In float64: the inputs are bf16, so products are exact and sums good to 2^-50.

struct SelectArgs {
  CacheView cache;
  const bf16_t* q;
  const int32_t *row_offsets, *lens;
  double* scores;                         // [rows][heads_kv][P]
  int32_t* pages;                         // [rows][heads_kv][n_sel]
  int B, H, G, total_rows, k_max, L_max, P, n_sel, n_first, n_last;
};

// Scores of 64 pages by one wave: D / 8 lanes a page, 16 bytes each, all loads in
// flight at once.  Returns the score of page j0 + `at`.  qs: the lane's eight features
// of the summed queries.
template <int D>
__device__ __forceinline__ double score64(const SelectArgs& a, int b, int hk, int j0, int vis,
                                          const double (&qs)[8], int& at) {
  constexpr int C = D / 8, PL = 64 / C, N = C;       // lanes a page, pages at a time, times
  const int lane = (int)__lane_id(), c = lane % C, pl = lane / C;
  const int mine = a.cache.page(b, min(j0 + lane, vis - 1));
  u32x4 x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int pg = max(__shfl(mine, PL * i + pl, kWave), 0);
    x[i] = *reinterpret_cast<const u32x4*>(
        a.cache.mean + ((size_t)(uint32_t)pg * a.cache.heads_kv + hk) * D + 8 * c);
  }
  double z[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    double y[8];
    unpack16_f64<bf16_t>(x[i], y);
    z[i] = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[i] = fma(qs[e], y[e], z[i]);
  }
  // sums over the lanes of a page; lane c keeps those of time c
#pragma unroll
  for (int m = N / 2; m >= 1; m >>= 1) {
    const bool up = (c & m) != 0;
#pragma unroll
    for (int i = 0; i < m; ++i) {
      const double keep = up ? z[i + m] : z[i], give = up ? z[i] : z[i + m];
      z[i] = keep + __shfl_xor(give, m, kWave);
    }
  }
  at = PL * c + pl;
  return __shfl(mine, at, kWave) < 0 ? 0.0 : z[0];
}
// The lane's features of the sum of a key head's queries.
template <int D>
__device__ __forceinline__ void sum_queries(const SelectArgs& a, int row, int hk,
                                            double (&qs)[8]) {
  const bf16_t* q = a.q + ((size_t)row * a.H + hk * a.G) * D + 8 * ((int)__lane_id() % (D / 8));
#pragma unroll
  for (int e = 0; e < 8; ++e) qs[e] = 0.0;
#pragma unroll 4
  for (int g = 0; g < a.G; ++g) {
    double x[8];
    unpack16_f64<bf16_t>(*reinterpret_cast<const u32x4*>(q + (size_t)g * D), x);
#pragma unroll
    for (int e = 0; e < 8; ++e) qs[e] += x[e];
  }
}

// Scores of 256 pages a workgroup, for few rows and many pages.
template <int D>
__global__ void __launch_bounds__(256)
cache_score_kernel(SelectArgs a) {
  const int row = blockIdx.z, hk = blockIdx.y, j0 = 64 * (4 * blockIdx.x + threadIdx.x / 64);
  CacheSeq s;
  const int b = seq_of_row(a.row_offsets, a.lens, a.B, a.total_rows, a.k_max, a.L_max, row, s);
  if (b < 0) return;
  const int t = s.len - s.n + row - s.r0;
  const int vis = t < 0 ? 0 : min((t >> a.cache.shift) + 1, a.P);
  if (j0 >= vis) return;
  double qs[8];
  sum_queries<D>(a, row, hk, qs);
  int at;
  const double z = score64<D>(a, b, hk, j0, vis, qs, at);
  if (j0 + at < vis) a.scores[((size_t)row * a.cache.heads_kv + hk) * a.P + j0 + at] = z;
}

// The selection of one row and key head by a wave, for up to 64 K pages: lane l holds
// pages l, 64 + l, ..  The kk-th largest key is found bit by bit from the top (the
// largest t that kk keys reach), with ballots for the counts.
template <int D, int K>
__global__ void __launch_bounds__(256)
cache_select_wave_kernel(SelectArgs a) {
  constexpr int C = D / 8, PL = 64 / C;
  const int lane = threadIdx.x & 63, hkv = a.cache.heads_kv;
  const int item = 4 * blockIdx.x + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = item / hkv, hk = item - row * hkv;
  if (row >= a.total_rows) return;
  CacheSeq s;
  const int b = seq_of_row(a.row_offsets, a.lens, a.B, a.total_rows, a.k_max, a.L_max, row, s);
  if (b < 0) return;
  const int t = s.len - s.n + row - s.r0;
  const int vis = t < 0 ? 0 : min((t >> a.cache.shift) + 1, a.P), kk = min(a.n_sel, vis);
  int32_t* out = a.pages + (size_t)item * a.n_sel;
  uint64_t key[K], taken[K];
#pragma unroll
  for (int i = 0; i < K; ++i) taken[i] = 0ull;
  if (vis <= a.n_sel) {                              // all of them
#pragma unroll
    for (int i = 0; i < K; ++i) taken[i] = __ballot(64 * i + lane < vis);
  } else {
    double qs[8];
    sum_queries<D>(a, row, hk, qs);
#pragma unroll
    for (int i = 0; i < K; ++i) {
      key[i] = 0;
      if (64 * i < vis) {
        int at;
        double z = score64<D>(a, b, hk, 64 * i, vis, qs, at);
        z = __shfl(z, (lane % PL) * C + lane / PL, kWave);       // of page 64 i + lane
        const int j = 64 * i + lane;
        key[i] = j >= vis ? 0ull : j < a.n_first || j >= vis - a.n_last ? ~0ull : order_key(z);
      }
    }
    uint64_t least = 0;                              // at least kk keys are not below it
    bool exact = false;
    for (int bit = 63; bit >= 0 && !exact; --bit) {
      const uint64_t next = least | 1ull << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < K; ++i) n += __popcll(__ballot(key[i] >= next));
      if (n >= kk) least = next;
      exact = n == kk;
    }
    int need = kk;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      taken[i] = __ballot(exact ? key[i] >= least : key[i] > least);
      need -= __popcll(taken[i]);
    }
    // (equal keys: the lowest pages)
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const uint64_t same = __ballot(key[i] == least && 64 * i + lane < vis);
      const bool mine = ((same >> lane) & 1) &&
                        __popcll(same & ((1ull << lane) - 1ull)) < need;
      const uint64_t more = exact ? 0ull : __ballot(mine);
      taken[i] |= more;
      need -= __popcll(more);
    }
  }
  int before = 0;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    if ((taken[i] >> lane) & 1)
      out[before + __popcll(taken[i] & ((1ull << lane) - 1ull))] = 64 * i + lane;
    before += __popcll(taken[i]);
  }
  for (int i = before + lane; i < a.n_sel; i += 64) out[i] = -1;
}

// The selection of one row and key head: scores (from the launch before, or made here
// and kept in LDS), their keys in registers, a radix select, and the chosen pages in
// ascending order, -1 behind them.
template <int D, int MAXPT, bool SCORED>
__global__ void __launch_bounds__(1024)
cache_select_kernel(SelectArgs a) {
  constexpr int THREADS = 1024;
  __shared__ SelectShared sh;
  __shared__ uint32_t scan[THREADS / 64 + 1];
  __shared__ double zs[SCORED ? 1 : THREADS * MAXPT];
  const int row = blockIdx.y, hk = blockIdx.x, tid = threadIdx.x;
  CacheSeq s;
  const int b = seq_of_row(a.row_offsets, a.lens, a.B, a.total_rows, a.k_max, a.L_max, row, s);
  if (b < 0) return;
  const int t = s.len - s.n + row - s.r0;
  const int vis = t < 0 ? 0 : min((t >> a.cache.shift) + 1, a.P);
  const double* z = a.scores + ((size_t)row * a.cache.heads_kv + hk) * a.P;
  int32_t* out = a.pages + ((size_t)row * a.cache.heads_kv + hk) * a.n_sel;
  if constexpr (!SCORED) {
    if (vis > a.n_sel) {                             // (else all of them)
      double qs[8];
      sum_queries<D>(a, row, hk, qs);
      for (int j0 = tid & ~63; j0 < vis; j0 += THREADS) {
        int at;
        const double x = score64<D>(a, b, hk, j0, vis, qs, at);
        if (j0 + at < vis) zs[j0 + at] = x;
      }
    }
    __syncthreads();
    z = zs;
  }
  const int C = (vis + THREADS - 1) / THREADS, e0 = tid * C, cnt = clampi(vis - e0, 0, C);
  uint64_t keys[MAXPT];
#pragma unroll
  for (int i = 0; i < MAXPT; ++i) {
    keys[i] = 0;
    const int j = e0 + i;
    if (i < cnt && vis > a.n_sel)
      keys[i] = j < a.n_first || j >= vis - a.n_last ? ~0ull : order_key(z[j]);
  }
  const int kk = min(a.n_sel, vis);
  const SelectMask<MAXPT> flags = block_select_top_wide<MAXPT>(keys, cnt, vis, kk, &sh);
  uint32_t total;
  uint32_t at = block_exclusive_scan((uint32_t)__popcll((uint64_t)flags), scan, &total);
#pragma unroll
  for (int i = 0; i < MAXPT; ++i)
    if ((flags >> i) & 1) out[at++] = e0 + i;
  for (int i = (int)total + tid; i < a.n_sel; i += THREADS) out[i] = -1;
}

// ---------------------------------------------------------------------------
// Launches

CacheView cache_view(const skip_kv_cache_t& c) {
  int shift = 5;
  while ((1 << shift) < c.page_tokens) ++shift;
  return CacheView{static_cast<bf16_t*>(c.k), static_cast<bf16_t*>(c.v),
                   static_cast<bf16_t*>(c.mean), c.page_table, (long long)c.n_pages, c.heads_kv,
                   c.pages_max, shift};
}

template <typename T, int D>
static hipError_t launch_append(const AppendArgs& a, long long slots, bool pieces, hipStream_t s) {
  const unsigned n = (unsigned)slots, hk = (unsigned)a.cache.heads_kv;
  if (!pieces) {
    cache_append_kernel<T, D, false><<<dim3(n, hk), kAppThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  const unsigned z = a.q ? (unsigned)((a.G + kAppHeads - 1) / kAppHeads) : 1u;
  cache_append_kernel<T, D, true>
      <<<dim3(n << (a.cache.shift - 5), hk, z), kAppThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.cache.mean) return e;
  cache_mean_kernel<D><<<dim3(n, hk), kAppThreads, 0, s>>>(a);
  return hipGetLastError();
}

// n tokens of a sequence go to at most n pages, and to n / page + 2
static long long append_slots(const skip_problem_t& p, const skip_kv_cache_t& c) {
  return std::min<long long>(p.total_kept, p.total_kept / c.page_tokens + 2ll * p.B);
}

bool cache_append_fits(const skip_problem_t& p, const skip_kv_cache_t& c) {
  return append_slots(p, c) < kMaxGrid;
}

hipError_t launch_cache_append(const skip_problem_t& p, const skip_kv_cache_t& c,
                               const skip_rotation_t* rot, const void* q, int64_t qs,
                               const void* k, int64_t ks, const void* v, int64_t vs,
                               const int32_t* row_offsets, const int32_t* lens,
                               const int32_t* positions, void* q_out, hipStream_t s) {
  AppendArgs a{cache_view(c), q, k, v, qs, ks, vs, rot ? rot->freq : nullptr, row_offsets, lens,
               positions, static_cast<bf16_t*>(q_out), p.B, p.H, p.H / c.heads_kv, p.total_kept,
               p.k_max, p.L_max, rot ? rot->dims / 2 : 0, rot ? rot->pairs : 0};
  const long long slots = append_slots(p, c);
  // Where many tokens make few such pages, 32 tokens and four heads a workgroup and the
  // means after them (6 prompts of 78 to 210 tokens, 16 heads over one, pages of 256: 70 us
  // by page, 13.6 so).
  const bool pieces = p.k_max > kAppTokens && c.page_tokens > kAppTokens &&
                      slots * c.heads_kv < 512;
  if (p.dtype == SKIP_F32)
    return p.d_h == 64 ? launch_append<float, 64>(a, slots, pieces, s)
                       : launch_append<float, 128>(a, slots, pieces, s);
  return p.d_h == 64 ? launch_append<bf16_t, 64>(a, slots, pieces, s)
                     : launch_append<bf16_t, 128>(a, slots, pieces, s);
}

static int select_pages(const skip_problem_t& p, const skip_kv_cache_t& c) {
  return (p.L_max + c.page_tokens - 1) / c.page_tokens;
}

bool cache_select_fits(const skip_problem_t& p, const skip_kv_cache_t& c) {
  return select_pages(p, c) <= 16384 && p.total_kept <= 65535 &&
         (long long)p.total_kept * c.heads_kv < 4 * kMaxGrid;
}

// Whether scores are made by a launch of their own, which takes more workgroups for
// few rows over many pages (8 rows and key heads of d_h 128: 1024 pages 11.2 us in one
// launch, 12.1 in two; 2048 pages 16.0 and 12.7; 256 of them over 1024 pages 12.4 and 17.7,
// 4096 pages 29.7 and 37.1).
static bool score_apart(const skip_problem_t& p, const skip_kv_cache_t& c) {
  return select_pages(p, c) > 1536 && (long long)p.total_kept * c.heads_kv < 256;
}

size_t cache_select_scratch(const skip_problem_t& p, const skip_kv_cache_t& c) {
  if (!score_apart(p, c)) return 0;
  return (size_t)p.total_kept * c.heads_kv * select_pages(p, c) * sizeof(double);
}

template <int D>
static hipError_t launch_select(const SelectArgs& a, bool apart, hipStream_t s) {
  const dim3 grid((unsigned)a.cache.heads_kv, (unsigned)a.total_rows);
  if (apart) {
    const dim3 g((unsigned)((a.P + 255) / 256), (unsigned)a.cache.heads_kv, (unsigned)a.total_rows);
    cache_score_kernel<D><<<g, 256, 0, s>>>(a);
    cache_select_kernel<D, 16, true><<<grid, 1024, 0, s>>>(a);
  } else if (a.P <= 256) {
    const unsigned g = (unsigned)(((long long)a.total_rows * a.cache.heads_kv + 3) / 4);
    if (a.P <= 64) cache_select_wave_kernel<D, 1><<<dim3(g), 256, 0, s>>>(a);
    else if (g >= 128) cache_select_wave_kernel<D, 4><<<dim3(g), 256, 0, s>>>(a);
    else cache_select_kernel<D, 2, false><<<grid, 1024, 0, s>>>(a);
  } else if (a.P <= 2048) {
    cache_select_kernel<D, 2, false><<<grid, 1024, 0, s>>>(a);
  } else {
    cache_select_kernel<D, 16, false><<<grid, 1024, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_cache_select(const skip_problem_t& p, const skip_kv_cache_t& c, const void* q,
                               const int32_t* row_offsets, const int32_t* lens, int n_sel,
                               int n_first, int n_last, int32_t* pages, void* scratch,
                               hipStream_t s) {
  SelectArgs a{cache_view(c), static_cast<const bf16_t*>(q), row_offsets, lens,
               static_cast<double*>(scratch), pages, p.B, p.H, p.H / c.heads_kv, p.total_kept,
               p.k_max, p.L_max, select_pages(p, c), n_sel, n_first, n_last};
  const bool apart = score_apart(p, c);
  return p.d_h == 64 ? launch_select<64>(a, apart, s) : launch_select<128>(a, apart, s);
}

}  // namespace skip
