// The join of partial results of the cache's attention (internal to libskip.so).
#pragma once

#include "skip_cache.h"

namespace skip {

constexpr float kCacheLn2 = 0.6931471805599453f;

// Joins the parts of each virtual row: of its prefix, then of its own tokens, in order.
// D / 4 lanes a virtual row.
// OWN: items of sequences' own tokens, of listed pages, or of the sequences with many
// new tokens.
enum JoinOf { kJoinOwn, kJoinListed, kJoinTall };
struct JoinArgs {
  CacheBatch batch;
  CacheResults res;
  void* O;
  float* lse;
  int listed_tiles;                 // of a row and key head
};
template <int D, bool OUT_F32, JoinOf OWN>
__global__ void __launch_bounds__(256)
cache_join_kernel(JoinArgs a) {
  constexpr int NC4 = D / 4, VR = 256 / NC4;       // lanes a virtual row, virtual rows
  const CacheBatch& bt = a.batch;
  const int hkv = bt.heads_kv, cols = a.res.cols_own;
  const int per_row = (bt.H + VR - 1) / VR;
  const int row = blockIdx.x / per_row;
  const int h = (blockIdx.x - row * per_row) * VR + threadIdx.x / NC4;
  const int c4 = threadIdx.x % NC4;
  CacheSeq s;
  const int b = seq_of_row(bt.row_offsets, bt.lens, bt.B, bt.total_rows, bt.k_max, bt.L_max, row, s);
  if (b < 0 || h >= bt.H) return;
  const int hk = h / bt.G, g = h - hk * bt.G;
  const size_t vr = (size_t)row * bt.H + h;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float4 x, float xm, float xl) {
    const float to = fmaxf(m, xm), ref = to == -INFINITY ? 0.f : to;
    const float f = __builtin_amdgcn_exp2f(m - ref), fx = __builtin_amdgcn_exp2f(xm - ref);
    o = make_float4(fmaf(x.x, fx, o.x * f), fmaf(x.y, fx, o.y * f), fmaf(x.z, fx, o.z * f),
                    fmaf(x.w, fx, o.w * f));
    l = fmaf(xl, fx, l * f);
    m = to;
  };
  // results of the tiles at places [first, first + nt), in column col of pc
  auto parts = [&](bool own, const float* part, int pc, int per, int first, int nt, int col) {
    const int c0 = first / per, c1 = (first + nt - 1) / per;
    if (c0 == c1) {                                // (alone: not reached)
      const float* w = whole_at<D>(a.res, bt, own, vr);
      add(*reinterpret_cast<const float4*>(w + 4 * c4), w[D], w[D + 1]);
      return;
    }
    constexpr int U = 8;                           // parts in flight
    for (int c = c0; c <= c1; c += U) {
      float4 x[U];
      float xm[U], xl[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int k = min(c + i, c1);
        const float* w = part + (size_t)(2 * k + (k == c0 ? 1 : 0)) *
                                    part_floats<D>(pc);
        x[i] = *reinterpret_cast<const float4*>(w + (size_t)col * D + 4 * c4);
        xm[i] = w[(size_t)pc * D + col];
        xl[i] = w[(size_t)pc * D + pc + col];
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (c + i <= c1) add(x[i], xm[i], xl[i]);
    }
  };
  const int32_t* pers = a.res.meta + (size_t)bt.B * kCacheMeta;
  int first, nt, col;
  bool alone = true;                               // no prefix
  if constexpr (OWN == kJoinListed) {
    nt = a.listed_tiles;
    first = (row * hkv + hk) * (nt + kOwnStart) + kOwnStart;
    col = g;
  } else if constexpr (OWN == kJoinTall) {
    const int v = (row - s.r0) * bt.G + g, rt = v / kPrefixRows;
    nt = SeqBlock::tall_tiles(bt, s.n, s.len, rt);
    first = hk * pers[1] + a.res.meta[(size_t)b * kCacheMeta] +
            SeqBlock::tall_before(bt, s.n, s.len, rt) + kPrefixStart;
    col = v % kPrefixRows;
  } else {
    const int4 x = reinterpret_cast<const int4*>(a.res.meta + (size_t)b * kCacheMeta)[0];
    const int4 y = reinterpret_cast<const int4*>(a.res.meta + (size_t)b * kCacheMeta)[1];
    const int P = x.z;
    alone = P == 0;
    if (!alone) {
      const int v = (row - x.w) * bt.G + g, n = SeqBlock::prefix_tiles(P);
      parts(false, a.res.part_pre, a.res.cols_pre, pers[1],
            x.y + kPrefixStart + (hk * SeqBlock::row_tiles(bt, y.x, kPrefixRows) +
                                  v / kPrefixRows) * (n + kPrefixStart), n, v % kPrefixRows);
    }
    const int v = (row - s.r0) * bt.G + g, lo = min(P, s.len);
    nt = SeqBlock::own_tiles(lo, s.len);
    first = x.x + kOwnStart +
            (hk * SeqBlock::row_tiles(bt, s.n, cols) + v / cols) * (nt + kOwnStart);
    col = v % cols;
  }
  const int per = pers[0];
  if (alone && first / per == (first + nt - 1) / per) return;          // (it is written)
  parts(true, a.res.part, cols, per, first, nt, col);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (OUT_F32)
    *reinterpret_cast<float4*>(static_cast<float*>(a.O) + vr * D + 4 * c4) =
        make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.O) + vr * D + 4 * c4) =
        make_uint2(pack2_bf16(o.x * inv, o.y * inv), pack2_bf16(o.z * inv, o.w * inv));
  if (a.lse && c4 == 0) a.lse[vr] = l == 0.f ? -INFINITY : (m + log2f(l)) * kCacheLn2;
}

template <int D, bool OUT_F32, JoinOf OWN>
inline hipError_t launch_join(const JoinArgs& a, hipStream_t s) {
  constexpr int VR = 1024 / D;
  const unsigned grid = (unsigned)a.batch.total_rows * (unsigned)((a.batch.H + VR - 1) / VR);
  cache_join_kernel<D, OUT_F32, OWN><<<dim3(grid), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace skip
