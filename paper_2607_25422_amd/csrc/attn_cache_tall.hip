// Attention of new tokens over a paged cache, for sequences with many of them and for
// shared prefixes: kernels and launches (the work of a workgroup is in
// skip_cache_tall.h).
#include <algorithm>

#include "skip_cache.h"
#include "skip_cache_join.h"
#include "skip_cache_rows.h"
#include "skip_cache_tall.h"
#include "skip_common.h"
#include "skip_internal.h"

namespace skip {

template <int D, bool OUT_F32, TallOf OF>
__global__ void __launch_bounds__(kTThreads, D == 64 ? 3 : 2)
cache_tall_kernel(TallArgs a) {
  __shared__ __attribute__((aligned(1024))) TallShared<D> sh;
  cache_tall_work<D, OUT_F32, OF>(a, sh, blockIdx.x);
}

// ---------------------------------------------------------------------------
// Launches

namespace {

struct TallPlan {
  int row_tiles, runs, cols;           // runs 0: an item a workgroup
  size_t meta, part;
};

TallPlan tall_plan(const skip_problem_t& p, const skip_kv_cache_t& c) {
  TallPlan x{};
  const long long G = p.H / c.heads_kv;
  x.row_tiles = (int)((p.k_max * G + kTRows - 1) / kTRows);
  // Few items are cut into equal runs (items as they come leave CUs without work: six
  // pieces of 98 to 129 rows over 3102 to 3362 tokens, 16 heads, 49 us in equal shares of each
  // item); about half a row tile of a sequence's is empty.
  const long long items = c.heads_kv * std::min<long long>(
      (long long)p.B * x.row_tiles, p.total_kept * G / kTRows + (p.B + 1) / 2);
  if (items < 2048 && x.row_tiles <= 64 && p.L_max > kTShort) {
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    x.runs = p.d_h == 64 ? 768 : 512;
    x.cols = (int)std::min<long long>(kTRows, (p.k_max * G + 31) / 32 * 32);
    x.meta = up(((size_t)p.B * kCacheMeta + 2) * sizeof(int32_t));
    x.part = 2 * (size_t)x.runs * x.cols * (p.d_h + 2) * sizeof(float);
  }
  return x;
}

}  // namespace

bool cache_tall(const skip_problem_t& p, const skip_kv_cache_t& c) {
  return (long long)p.k_max * (p.H / c.heads_kv) > 32;
}

size_t cache_tall_scratch(const skip_problem_t& p, const skip_kv_cache_t& c) {
  const TallPlan x = tall_plan(p, c);
  return x.meta + x.part;
}

template <int D, bool OUT_F32>
static hipError_t launch_tall(const TallArgs& a, hipStream_t s) {
  if (a.runs == 0) {
    const unsigned grid = (unsigned)a.batch.B * a.batch.heads_kv * a.row_tiles;
    cache_tall_kernel<D, OUT_F32, kTallItems><<<dim3(grid), kTThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  cache_tall_kernel<D, OUT_F32, kTallRuns><<<dim3(a.runs), kTThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_join<D, OUT_F32, kJoinTall>(JoinArgs{a.batch, a.res, a.O, a.lse, 0}, s);
}

hipError_t launch_cache_tall(const skip_problem_t& p, const skip_kv_cache_t& c, const void* q,
                             const int32_t* row_offsets, const int32_t* lens, void* O, float* lse,
                             void* scratch, hipStream_t s) {
  const TallPlan x = tall_plan(p, c);
  CacheResults res{};
  if (x.runs) {
    res.meta = static_cast<int32_t*>(scratch);
    res.part = reinterpret_cast<float*>(static_cast<char*>(scratch) + x.meta);
    res.cols_own = x.cols;
  }
  TallArgs a{cache_batch(p, c, row_offsets, lens, nullptr, nullptr), cache_view(c), res,
             static_cast<const bf16_t*>(q), O, lse, x.row_tiles, x.runs,
             p.B * c.heads_kv % 8 == 0, p.sm_scale * 1.4426950408889634f};
  if (p.d_h == 64) return p.o_f32 ? launch_tall<64, true>(a, s) : launch_tall<64, false>(a, s);
  return p.o_f32 ? launch_tall<128, true>(a, s) : launch_tall<128, false>(a, s);
}

// Prefixes, then sequences' own tokens, by the same workgroups: those that are through
// with their run of one take theirs of the other.
template <int D, int R, bool OUT_F32>
__global__ void __launch_bounds__(kTThreads, 2)
cache_shared_kernel(TallArgs pre, CacheAttnArgs own) {
  constexpr size_t A = sizeof(TallShared<D>), B = sizeof(RowsShared<D, R>);
  __shared__ __attribute__((aligned(1024))) uint8_t lds[A > B ? A : B];
  cache_tall_work<D, OUT_F32, kTallPrefixes>(pre, *reinterpret_cast<TallShared<D>*>(lds),
                                             blockIdx.x);
  __syncthreads();                                  // (the prefix's tiles are read)
  cache_rows<D, R, OUT_F32, false, false>(own, *reinterpret_cast<RowsShared<D, R>*>(lds),
                                          blockIdx.x);
}

hipError_t launch_cache_shared(const CacheAttnArgs& own, int d_h, int R, hipStream_t s) {
  TallArgs pre{own.batch, own.cache, own.res, own.q, nullptr, nullptr, 0, kPrefixRuns, 0,
               own.scale_log2};
  static_assert(kTThreads == kCThreads, "one launch of both");
  const dim3 grid(kPrefixRuns);
  const int form = (d_h == 128 ? 4 : 0) + (R == 2 ? 2 : 0) + (own.o_f32 ? 1 : 0);
  switch (form) {
    case 0: cache_shared_kernel<64, 1, false><<<grid, kTThreads, 0, s>>>(pre, own); break;
    case 1: cache_shared_kernel<64, 1, true><<<grid, kTThreads, 0, s>>>(pre, own); break;
    case 2: cache_shared_kernel<64, 2, false><<<grid, kTThreads, 0, s>>>(pre, own); break;
    case 3: cache_shared_kernel<64, 2, true><<<grid, kTThreads, 0, s>>>(pre, own); break;
    case 4: cache_shared_kernel<128, 1, false><<<grid, kTThreads, 0, s>>>(pre, own); break;
    case 5: cache_shared_kernel<128, 1, true><<<grid, kTThreads, 0, s>>>(pre, own); break;
    case 6: cache_shared_kernel<128, 2, false><<<grid, kTThreads, 0, s>>>(pre, own); break;
    default: cache_shared_kernel<128, 2, true><<<grid, kTThreads, 0, s>>>(pre, own); break;
  }
  return hipGetLastError();
}

}  // namespace skip
