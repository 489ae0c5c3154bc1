// Attention of new tokens over a paged cache: kernels and launches (the work of a
// workgroup is in skip_cache_rows.h, that of sequences with many new tokens in
// skip_cache_tall.h).
#include <algorithm>

#include "skip_cache.h"
#include "skip_cache_join.h"
#include "skip_cache_rows.h"
#include "skip_common.h"
#include "skip_internal.h"

namespace skip {

template <int D, int R, bool OUT_F32, bool LISTED, bool SOLO>
__global__ void __launch_bounds__(kCThreads, D == 64 && R == 1 ? 3 : 2)
cache_attn_kernel(CacheAttnArgs a) {
  __shared__ __attribute__((aligned(16))) RowsShared<D, R> sh;
  cache_rows<D, R, OUT_F32, LISTED, SOLO>(a, sh, blockIdx.x);
}

// ---------------------------------------------------------------------------
// Launches

namespace {

struct CachePlan {
  int R, runs, cols_pre;
  bool direct, solo, prefixes;
  size_t meta, part, part_pre, whole;          // bytes
};

CachePlan cache_plan(const skip_problem_t& p, const skip_kv_cache_t& c, int n_sel, bool prefixes) {
  CachePlan x{};
  const int G = p.H / c.heads_kv;
  if (n_sel > 0) {
    // many short items: a wave each
    const int pages = std::min(n_sel, (p.L_max + c.page_tokens - 1) / c.page_tokens);
    const int nt = pages * (c.page_tokens / kCTile), items = p.total_kept * c.heads_kv;
    x.R = G <= 16 ? 1 : 2;
    x.direct = nt <= 16 || items >= 512;
    x.solo = x.direct && items >= 1024 && nt <= 64;
    const int side = x.solo ? kCWaves : 1;
    x.runs = !x.direct ? 512 : 8 * (((items + 7) / 8 + side - 1) / side);
  } else {
    // sequences of up to 512 tokens: an item a workgroup, prefixes with them.  Prefixes
    // of their own take a launch more: where all sequences' keys and values are 64 MB
    // or more (9 sequences of 600 tokens, one key head: 29 us with it, 13 without)
    x.direct = p.L_max <= 512;
    x.prefixes = prefixes && !x.direct &&
                 4ll * p.B * c.heads_kv * p.L_max * p.d_h >= (64ll << 20);
    x.R = p.k_max * G <= 16 ? 1 : 2;
    const int cols = 16 * x.R;
    x.runs = x.direct ? p.B * c.heads_kv * ((p.k_max * G + cols - 1) / cols) : 512;
  }
  if (!x.direct) {
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    x.meta = up(((size_t)p.B * kCacheMeta + 2) * sizeof(int32_t));
    x.part = up(2 * (size_t)x.runs * 16 * x.R * (p.d_h + 2) * sizeof(float));
    if (x.prefixes) {
      x.cols_pre = (int)std::min<long long>(kPrefixRows, ((long long)p.total_kept * G + 31) / 32 * 32);
      x.part_pre = up(2 * (size_t)kPrefixRuns * x.cols_pre * (p.d_h + 2) * sizeof(float));
      x.whole = 2 * (size_t)p.total_kept * p.H * (p.d_h + 4) * sizeof(float);
    }
  }
  return x;
}

template <int D, int R, bool OUT_F32, bool LISTED>
hipError_t launch_one(const CacheAttnArgs& a, bool solo, hipStream_t s) {
  const dim3 grid((unsigned)a.runs);
  hipError_t e;
  if (a.batch.prefix_ids) {
    e = launch_cache_shared(a, D, R, s);
    if (e != hipSuccess) return e;
    return launch_join<D, OUT_F32, kJoinOwn>(JoinArgs{a.batch, a.res, a.O, a.lse, 0}, s);
  }
  if (LISTED && solo) cache_attn_kernel<D, R, OUT_F32, true, true><<<grid, kCThreads, 0, s>>>(a);
  else cache_attn_kernel<D, R, OUT_F32, LISTED, false><<<grid, kCThreads, 0, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || a.direct) return e;
  const JoinArgs j{a.batch, a.res, a.O, a.lse, a.n_sel * (1 << a.cache.shift) / kCTile};
  return launch_join<D, OUT_F32, LISTED ? kJoinListed : kJoinOwn>(j, s);
}
template <int D, bool LISTED>
hipError_t launch_rows(const CacheAttnArgs& a, const CachePlan& x, hipStream_t s) {
  if (x.R == 1)
    return a.o_f32 ? launch_one<D, 1, true, LISTED>(a, x.solo, s)
                   : launch_one<D, 1, false, LISTED>(a, x.solo, s);
  return a.o_f32 ? launch_one<D, 2, true, LISTED>(a, x.solo, s)
                 : launch_one<D, 2, false, LISTED>(a, x.solo, s);
}

}  // namespace

// Tiles are counted in 32 bits (with the workgroups' shares rounded up), and a grid has
// fewer than 2^32 threads.
bool cache_attn_fits(const skip_problem_t& p, const skip_kv_cache_t& c, int n_sel) {
  const long long G = p.H / c.heads_kv, hkv = c.heads_kv, rows = p.total_kept;
  const long long items = n_sel > 0 ? rows * hkv : (rows * G / 16 + 2ll * p.B) * hkv;
  const long long tiles = kOwnStart + (n_sel > 0 ? (long long)n_sel * (c.page_tokens / kCTile)
                                                 : p.L_max / kCTile + 2);
  const long long cols = n_sel == 0 && cache_tall(p, c) ? kPrefixRows : 16;
  return items <= (1ll << 30) / tiles && rows * ((p.H + 7) / 8) < kMaxGrid &&
         (n_sel > 0 ? items : p.B * hkv * ((p.k_max * G + cols - 1) / cols)) < kMaxGrid;
}

size_t cache_attn_scratch(const skip_problem_t& p, const skip_kv_cache_t& c, int n_sel,
                          bool prefixes) {
  if (n_sel == 0 && cache_tall(p, c)) return cache_tall_scratch(p, c);
  const CachePlan x = cache_plan(p, c, n_sel, prefixes);
  return x.meta + x.part + x.part_pre + x.whole;
}

hipError_t launch_cache_attn(const skip_problem_t& p, const skip_kv_cache_t& c, const void* q,
                             const int32_t* row_offsets, const int32_t* lens,
                             const int32_t* prefix_ids, const int32_t* prefix_lens,
                             const int32_t* pages, int n_sel, void* O, float* lse, void* scratch,
                             hipStream_t s) {
  if (n_sel == 0 && cache_tall(p, c))
    return launch_cache_tall(p, c, q, row_offsets, lens, O, lse, scratch, s);
  const CachePlan x = cache_plan(p, c, n_sel, prefix_ids != nullptr);
  char* w = static_cast<char*>(scratch);
  auto take = [&](size_t bytes) {
    char* r = w;
    w += bytes;
    return reinterpret_cast<float*>(r);
  };
  CacheResults res{};
  if (!x.direct) {
    res.meta = reinterpret_cast<int32_t*>(take(x.meta));
    res.part = take(x.part);
    res.part_pre = take(x.part_pre);
    res.whole = take(x.whole);
    res.cols_own = 16 * x.R;
    res.cols_pre = x.cols_pre;
  }
  CacheAttnArgs a{cache_batch(p, c, row_offsets, lens, x.prefixes ? prefix_ids : nullptr,
                              prefix_lens),
                  cache_view(c), res, static_cast<const bf16_t*>(q), pages, O, lse, n_sel, p.o_f32,
                  x.runs, x.direct, p.sm_scale * kCLog2e};
  if (n_sel > 0)
    return p.d_h == 64 ? launch_rows<64, true>(a, x, s) : launch_rows<128, true>(a, x, s);
  return p.d_h == 64 ? launch_rows<64, false>(a, x, s) : launch_rows<128, false>(a, x, s);
}

}  // namespace skip
