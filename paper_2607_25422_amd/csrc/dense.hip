// The layer after the attention (Alg. 1 hands the fused rows, with the kept
// tokens' skip connection, to the next layers): for every row r
//
//   Y[r] = act(W x_r + b) + R[r]
//
// bf16 rows and weights, float32 sums on v_mfma_f32_32x32x16_bf16; bias,
// activation and residual are float32 on the sums, and the result is rounded
// once.  x_r and R[r] are rows as given, or rows of [B][N][.] read through the
// kept indices.  Weights are packed as for the projections (proj.hip) with rows of
// zeros up to a multiple of 256.
//
//   dense_tile_kernel : 32 MB rows x 256 columns a workgroup
//   dense_rows_kernel : up to 32 rows x 64 columns, the contraction split over the
//                       workgroup's waves
//   dense_join_kernel : adds the parts of a contraction that several workgroups
//                       shared, in their order, and finishes
#include <algorithm>

#include "skip_common.h"
#include "skip_internal.h"

namespace skip {

constexpr int kDnNT = 256;         // columns of a packed tile
constexpr int kDnKS = 32;          // contraction of a packed step
constexpr int kDnStep = 64;        // contraction per step of dense_tile_kernel
constexpr int kDnThreads = 256;    // dense_tile_kernel: four waves of 64 columns
constexpr int kDnWaves = 8;        // dense_rows_kernel
constexpr long long kDnCUs = 256;

struct DenseArgs {
  const bf16_t* rows;
  const int32_t* rows_idx;         // NULL: row r is r
  const int32_t* kept_offsets;
  int B, N, M, d, d_out;
  const u32x4* Wp;
  const float* bias;
  const bf16_t* residual;
  const int32_t* residual_idx;
  int act, out_f32;
  void* Y;
  int splits;                      // parts of the contraction
  float* part;                     // [splits][M][d_out], where splits > 1
  int n_items;
};

// Row that a kept row r stands for: itself, or the row of [B][N] of its index.
__device__ __forceinline__ size_t dense_row(const DenseArgs& a, const int32_t* idx, int r) {
  if (!idx) return (size_t)r;
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (clampi(a.kept_offsets[mid], 0, a.M) <= r) lo = mid;
    else hi = mid;
  }
  return (size_t)lo * a.N + clampi(idx[r], 0, a.N - 1);
}

// x / 2 erfc(-x / sqrt 2).  With z = |x| / sqrt 2, erfc(z) = exp(-z^2) P(1 / (1 + p z)),
// P a polynomial fitted to exp(z^2) erfc(z) on 0 <= z <= 6 by weighted least squares
// (2.6e-7 relative); for x > 0 the rest of x.  Six times fewer instructions than the
// library's erfc, which took 45 us of 111 on 4616 rows of 4096 columns.  Relative error
// below zero: the exponent's two roundings and its constant's leave 1.25 x^2 2^-24, with
// the rest at most (1.25 x^2 + 16) 2^-24 down to x = -8.4 (measured: 6e-7
// above -2, 3e-6 above -8.4); from there on, where the result is below 2^-50, the
// polynomial's 4.5e-5.
__device__ __forceinline__ float gelu(float x) {
  constexpr float p = 0.3625f;
  const float ax = fabsf(x);
  const float t = __builtin_amdgcn_rcpf(fmaf(ax, p * 0.70710678f, 1.f));
  float h = -0.16227377519580077f;
  h = fmaf(h, t, 0.5469444163308744f);
  h = fmaf(h, t, -0.3379855943955391f);
  h = fmaf(h, t, 0.42285832312829363f);
  h = fmaf(h, t, 0.1080726978837203f);
  h = fmaf(h, t, 0.21891024798015968f);
  h = fmaf(h, t, 0.2034739364192221f);
  // (-z^2 log2 e)
  const float q = 0.5f * h * t * __builtin_amdgcn_exp2f(ax * ax * -0.72134752044448170f);
  const float m = fminf(ax, 1e3f);  // (infinity times q = 0 is no number)
  return x < 0.f ? -m * q : fmaf(-m, q, x);
}
// x / (1 + exp(-x))
__device__ __forceinline__ float silu(float x) {
  return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
}

// Eight sums of a row, columns j .. j + 7: bias, activation, residual (both given
// as loaded; zeros where there is none), store at element `at` of Y.
__device__ __forceinline__ void dense_finish8(const DenseArgs& a, size_t at, const float (&b)[8],
                                              const u32x4& res, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] += b[e];
  if (a.act == SKIP_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = gelu(x[e]);
  } else if (a.act == SKIP_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = silu(x[e]);
  } else if (a.act == SKIP_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] < 0.f ? 0.f : x[e];  // keeps NaN
  }
  float y[8];
  unpack8_bf16(res, y);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] += y[e];
  if (a.out_f32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(a.Y) + at);
    o[0] = make_float4(x[0], x[1], x[2], x[3]);
    o[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(a.Y) + at) =
        u32x4{pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]), pack2_bf16(x[4], x[5]),
              pack2_bf16(x[6], x[7])};
  }
}
__device__ __forceinline__ void dense_bias8(const DenseArgs& a, int j, float (&b)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = 0.f;
  if (a.bias && j < a.d_out) {
    const float4 b0 = reinterpret_cast<const float4*>(a.bias + j)[0];
    const float4 b1 = reinterpret_cast<const float4*>(a.bias + j)[1];
    b[0] = b0.x; b[1] = b0.y; b[2] = b0.z; b[3] = b0.w;
    b[4] = b1.x; b[5] = b1.y; b[6] = b1.z; b[7] = b1.w;
  }
}
__device__ __forceinline__ u32x4 dense_residual8(const DenseArgs& a, size_t row, int j) {
  return a.residual ? *reinterpret_cast<const u32x4*>(a.residual + row * a.d_out + j)
                    : u32x4{0u, 0u, 0u, 0u};
}
__device__ __forceinline__ void dense_finish_at(const DenseArgs& a, int r, int j, float (&x)[8]) {
  float b[8];
  dense_bias8(a, j, b);
  const u32x4 res = dense_residual8(a, dense_row(a, a.residual_idx, r), j);
  dense_finish8(a, (size_t)r * a.d_out + j, b, res, x);
}
// The same sums as a part of the contraction.
__device__ __forceinline__ void dense_part8(const DenseArgs& a, int split, int r, int j,
                                            const float (&x)[8]) {
  float4* o = reinterpret_cast<float4*>(a.part + ((size_t)split * a.M + r) * a.d_out + j);
  o[0] = make_float4(x[0], x[1], x[2], x[3]);
  o[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Packed order as in proj.hip (column tile, wave, step, k16 sub-step, lane: 16
// bytes of W), rows of W past d_out as zeros.
__global__ void __launch_bounds__(256)
dense_pack_kernel(const bf16_t* __restrict__ W, int d, int d_out, int tiles,
                  u32x4* __restrict__ Wp) {
  const size_t total = (size_t)tiles * kDnNT * d / 8;
  const int ksteps = d / kDnKS;
  for (size_t u = (size_t)blockIdx.x * blockDim.x + threadIdx.x; u < total;
       u += (size_t)gridDim.x * blockDim.x) {
    const int l = (int)(u % 64);
    size_t r = u / 64;
    const int kk = (int)(r % 2); r /= 2;
    const int s = (int)(r % ksteps); r /= ksteps;
    const int j = (int)r * 32 + (l & 31);
    const int col = s * kDnKS + (2 * kk + (l >> 5)) * 8;
    Wp[u] = j < d_out ? *reinterpret_cast<const u32x4*>(W + (size_t)j * d + col)
                      : u32x4{0u, 0u, 0u, 0u};
  }
}

// Workgroup: 32 MB rows x 256 columns, a part of the contraction, in steps of 64 (a
// row's 128 bytes of a step are one cache line).  The row tile arrives in a
// three-slot LDS ring by direct global->LDS loads two steps ahead and is published
// one step early; each wave's weights come from the packed copy into registers WD
// steps ahead, one coalesced run a load: they are used by this wave alone, so LDS
// would only add a way.  Items are dealt to the XCDs in runs, row tile fastest, so
// that the items of one XCD share their weights in its L2.
//
// 3088 rows of 4096 by 4096 columns take 93 us in a graph of such calls, 98 to 101 with
// a residual and inputs from HBM (1.04 PF; products alone, fed with the same data from
// registers, 1.74 PF, and 1.44 with one operand from LDS, where the card's power limit
// lowers the clock).  The matrix units are 43 % busy: 224 items leave 32 of 256 CUs idle,
// one workgroup a CU is one wave a SIMD, its operand reads meet bank conflicts (4.3 cycles
// each), and a start and end take 4 + 1.1 us a block of 32 rows; with MB <= 4 and one
// step of weights ahead, two workgroups fit a CU and hide most of that (4616 rows of 1408
// by 4096: MB = 4 62 us, 5 to 8 66, 72, 78 and 92).
template <int MB>
__global__ void __launch_bounds__(kDnThreads, MB <= 4 ? 2 : 1)
dense_tile_kernel(DenseArgs a) {
  constexpr int NB = 2, SUB = kDnStep / 16;           // k16 sub-steps of a step
  constexpr int RING = 3, AH = 2, WD = MB <= 4 ? 1 : 2;
  constexpr int MT = 32 * MB, A_ELEMS = MT * kDnStep;
  constexpr int NI = MB;                              // direct loads of a row tile per wave
  constexpr int PITCH = 72;                           // floats of a row in the epilogue
  __shared__ __attribute__((aligned(1024))) union {
    bf16_t ring[RING * A_ELEMS];
    float out[4][32 * PITCH];
  } sh;
  __shared__ int sh_row[MT], sh_res[MT];

  const int per_xcd = gridDim.x / 8;
  int item = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (item >= a.n_items) return;
  const int MTL = (a.M + MT - 1) / MT;
  const int mt = item % MTL;
  item /= MTL;
  const int split = item % a.splits, nt = item / a.splits;
  const int i0 = mt * MT, j0 = nt * kDnNT;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int k32 = a.d / kDnKS;                        // packed steps of 32
  const int odd = k32 & 1, all_steps = k32 / 2;       // (a first half step of its own)
  const int s_begin = (int)((long long)all_steps * split / a.splits);
  const int steps = (int)((long long)all_steps * (split + 1) / a.splits) - s_begin;
  const int hh = lane >> 5, r32 = lane & 31;

  // the lane's 16-byte chunks of a row tile: chunk g is row g / 8, physical
  // chunk g % 8 holding logical chunk (g % 8) ^ row % 8 (the operand reads of 8
  // consecutive rows hit distinct banks)
  // (the rows that kept rows stand for are looked up once)
  if (tid < MT) {
    const int r = min(i0 + tid, a.M - 1);
    sh_row[tid] = (int)dense_row(a, a.rows_idx, r);
    sh_res[tid] = (int)dense_row(a, a.residual_idx, r);
  }
  __syncthreads();
  const bf16_t* asrc[NI];
#pragma unroll
  for (int q = 0; q < NI; ++q)
    asrc[q] = a.rows + (size_t)sh_row[(wave * NI + q) * 8 + (lane >> 3)] * a.d;
  const int acol = odd * kDnKS + s_begin * kDnStep + ((lane & 7) ^ ((lane >> 3) & 7)) * 8;
  const uint32_t ar_lds = lds_addr(sh.ring) + (uint32_t)(wave * NI * 1024);
  auto issue_a = [&](int s) {
#pragma unroll
    for (int q = 0; q < NI; ++q)
      lds_dma16(asrc[q] + acol + s * kDnStep, __builtin_amdgcn_readfirstlane(
                                   ar_lds + ((uint32_t)s % RING) * (A_ELEMS * 2) + q * 1024));
  };
  const u32x4* wsrc = a.Wp + (size_t)(nt * 8 + wave * NB) * k32 * 128 + lane;
  const size_t wblk = (size_t)k32 * 128;              // from one 32-column block to the next
  auto load_w = [&](int s, int kk, u32x4 (&w)[NB]) {
    const size_t at = (size_t)(odd + 2 * (s_begin + s)) * 128 + kk * 64;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) w[nb] = wsrc[nb * wblk + at];
  };

  f32x16_t acc[NB][MB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[nb][mb][v] = 0.f;

  int aoff[SUB];
#pragma unroll
  for (int kk = 0; kk < SUB; ++kk) aoff[kk] = r32 * kDnStep + (((2 * kk + hh) ^ (r32 & 7)) << 3);
  auto read_a = [&](int s, int kk, u32x4 (&x)[MB]) {
    const bf16_t* At = sh.ring + ((uint32_t)s % RING) * A_ELEMS + aoff[kk];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
      x[mb] = *reinterpret_cast<const u32x4*>(At + mb * 32 * kDnStep);
  };
  // products of one sub-step, one operand read of the next beside each of the
  // first of them
  auto multiply = [&](const u32x4 (&x)[MB], const u32x4 (&w)[NB]) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) acc[nb][mb] = mfma32_bf16(x[mb], w[nb], acc[nb][mb]);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, MB * NB - MB, 0);
    __builtin_amdgcn_sched_barrier(0);
  };

  if (odd && split == 0) {
    // the first 32 columns, operands straight from memory
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 x[MB], w[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) w[nb] = wsrc[nb * wblk + kk * 64];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
        x[mb] = *reinterpret_cast<const u32x4*>(
            a.rows + (size_t)sh_row[mb * 32 + r32] * a.d + kk * 16 + hh * 8);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[nb][mb] = mfma32_bf16(x[mb], w[nb], acc[nb][mb]);
    }
  }
  if (steps > 0) {
#pragma unroll
    for (int q = 0; q < AH; ++q)
      if (q < steps) issue_a(q);
  }
  const int lw = max(steps - 1, 0);                   // (without a step: weights not multiplied)
  u32x4 w[WD][SUB][NB];
  if (all_steps > 0) {
#pragma unroll
    for (int u = 0; u < WD; ++u)
#pragma unroll
      for (int kk = 0; kk < SUB; ++kk) load_w(min(u, lw), kk, w[u][kk]);
  }
  wait_vmcnt<0>();
  barrier_nofence();
  u32x4 f[2][MB];
  read_a(0, 0, f[0]);

  // Step s: wait for this wave's part of the row tile of step s+1 (issued after
  // it: the weights of one step), barrier (publishes that tile; the slot of step
  // s-1 is free), request the tile of step s+2, multiply step s and read the first
  // operands of step s+1 (past the last step: stale values that nothing uses).
  auto step = [&](int s, u32x4 (&w)[SUB][NB]) {
    wait_vmcnt<SUB * NB>();
    barrier_nofence();
    if (s + AH < steps) issue_a(s + AH);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < SUB; ++kk) {
      if (kk + 1 < SUB) read_a(s, kk + 1, f[(kk + 1) & 1]);
      else read_a(s + 1, 0, f[0]);
      multiply(f[kk & 1], w[kk]);
      // unconditional (the last steps reload the final fragments): a conditional
      // load would make the compiler drain the queue before the next use of w
      load_w(min(s + WD, lw), kk, w[kk]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int s = 0;
  for (; s + WD <= steps; s += WD) {
#pragma unroll
    for (int u = 0; u < WD; ++u) step(s + u, w[u]);
  }
  if (s < steps) step(s, w[0]);

  // Accumulator element v of block (nb, mb) is row mb*32 + 8*(v/4) + 4*hh + v%4,
  // column 64*wave + 32*nb + r32: through the wave's own LDS, 32 rows at a time,
  // so that a lane finishes eight columns of a row
  __syncthreads();                                    // the ring is read
  float* out = sh.out[wave];
  const int j = j0 + 64 * wave + 8 * (lane & 7);
  float bias[8];
  dense_bias8(a, j, bias);
  unrolled<MB>([&](auto mb_) {
    constexpr int mb = decltype(mb_)::value;
    u32x4 res[4];                                     // in flight during the exchange
#pragma unroll
    for (int q = 0; q < 4; ++q)
      res[q] = j < a.d_out ? dense_residual8(a, (size_t)sh_res[mb * 32 + 8 * q + (lane >> 3)], j)
                           : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        out[(8 * (v >> 2) + 4 * hh + (v & 3)) * PITCH + 32 * nb + r32] = acc[nb][mb][v];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int lr = 8 * q + (lane >> 3), r = i0 + mb * 32 + lr;
      float x[8];
      *reinterpret_cast<float4*>(x) =
          *reinterpret_cast<const float4*>(out + lr * PITCH + 8 * (lane & 7));
      *reinterpret_cast<float4*>(x + 4) =
          *reinterpret_cast<const float4*>(out + lr * PITCH + 8 * (lane & 7) + 4);
      if (r < a.M && j < a.d_out) {
        if (a.splits > 1) dense_part8(a, split, r, j, x);
        else dense_finish8(a, (size_t)r * a.d_out + j, bias, res[q], x);
      }
    }
    __builtin_amdgcn_wave_barrier();
  });
}

// Few rows: bound by the weights' way from memory, so every wave streams its own
// part of them (64 columns, an eighth of the workgroup's contraction) straight
// into registers, a batch of loads ahead of the products; the rows come from the
// L2.  The waves' sums meet in LDS, added in wave order.  One row of 1024 by 1024
// columns takes 5.9 us, where the weights alone would take 0.3.
__global__ void __launch_bounds__(64 * kDnWaves, 2)
dense_rows_kernel(DenseArgs a) {
  constexpr int NB = 2, U = 4;                        // k16 groups a batch
  __shared__ float red[kDnWaves][16][64];
  const int per_xcd = gridDim.x / 8;
  const int item = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (item >= a.n_items) return;
  const int split = item % a.splits, ct = item / a.splits;
  const int j0 = ct * 64;
  const int lane = threadIdx.x & 63, hh = lane >> 5, r32 = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.d / 16, parts = a.splits * kDnWaves, me = split * kDnWaves + wv;
  const int g0 = (int)((long long)me * G / parts), g1 = (int)((long long)(me + 1) * G / parts);
  const int gl = max(g1 - 1, 0);

  const bf16_t* ap = a.rows + dense_row(a, a.rows_idx, min(r32, a.M - 1)) * a.d + hh * 8;
  const u32x4* wp = a.Wp + (size_t)ct * 2 * G * 64 + lane;
  struct Batch {
    u32x4 x[U], w[U][NB];
  };
  auto load = [&](Batch& b, int g) {                  // groups past the wave's are not multiplied
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t gg = (size_t)min(g + u, gl);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) b.w[u][nb] = wp[((size_t)nb * G + gg) * 64];
      b.x[u] = *reinterpret_cast<const u32x4*>(ap + gg * 16);
    }
  };
  f32x16_t acc[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[nb][v] = 0.f;
  auto multiply = [&](const Batch& b, int g) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + u < g1)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[nb] = mfma32_bf16(b.x[u], b.w[u][nb], acc[nb]);
  };
  Batch b0, b1;
  load(b0, g0);
  for (int g = g0; g < g1; g += 2 * U) {
    load(b1, g + U);
    multiply(b0, g);
    load(b0, g + 2 * U);
    multiply(b1, g + U);
  }
  // Element v of a block is row 8*(v/4) + 4*hh + v%4, column r32.  Blocks one
  // after the other: a thread of the first 128 adds the waves' sums of eight columns
  // of a row
  unrolled<NB>([&](auto nb_) {
    constexpr int nb = decltype(nb_)::value;
    if (nb > 0) __syncthreads();
#pragma unroll
    for (int v = 0; v < 16; ++v) red[wv][v][lane] = acc[nb][v];
    __syncthreads();
    if (threadIdx.x < 128) {
      const int r = threadIdx.x >> 2, c8 = (threadIdx.x & 3) * 8;
      const int v = 4 * (r >> 3) + (r & 3), l = 32 * ((r >> 2) & 1) + c8;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = red[0][v][l + e];
#pragma unroll
        for (int u = 1; u < kDnWaves; ++u) x[e] += red[u][v][l + e];
      }
      const int j = j0 + nb * 32 + c8;
      if (r < a.M && j < a.d_out) {
        if (a.splits > 1) dense_part8(a, split, r, j, x);
        else dense_finish_at(a, r, j, x);
      }
    }
  });
}

// Sum of the parts in their order, and the rest of the layer.
__global__ void __launch_bounds__(256)
dense_join_kernel(DenseArgs a) {
  const int c8 = a.d_out / 8;
  const size_t n = (size_t)a.M * c8;
  for (size_t u = (size_t)blockIdx.x * 256 + threadIdx.x; u < n; u += (size_t)gridDim.x * 256) {
    const int r = (int)(u / c8), j = (int)(u % c8) * 8;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) {
      const float4* p = reinterpret_cast<const float4*>(a.part + ((size_t)s * a.M + r) * a.d_out + j);
      const float4 y0 = p[0], y1 = p[1];
      x[0] += y0.x; x[1] += y0.y; x[2] += y0.z; x[3] += y0.w;
      x[4] += y1.x; x[5] += y1.y; x[6] += y1.z; x[7] += y1.w;
    }
    dense_finish_at(a, r, j, x);
  }
}

// ---------------------------------------------------------------------------
size_t dense_packed_bytes(int d, int d_out) {
  return (size_t)((d_out + kDnNT - 1) / kDnNT) * kDnNT * d * sizeof(bf16_t);
}

hipError_t launch_dense_pack(int d, int d_out, const void* W, void* packed, hipStream_t s) {
  hipLaunchKernelGGL(dense_pack_kernel, dim3(1024), dim3(256), 0, s, (const bf16_t*)W, d, d_out,
                     (d_out + kDnNT - 1) / kDnNT, static_cast<u32x4*>(packed));
  return hipGetLastError();
}

struct DenseShape {
  bool rows;             // dense_rows_kernel
  int mb, splits;
};
static DenseShape dense_shape(int M, int d, int d_out) {
  DenseShape s;
  if (M <= 32) {
    // One block of rows, up to as many parts as fill the chip once (a second round of
    // a few workgroups costs more than it brings: 1 x 16384 x 4104 in 3 parts 25 us,
    // in 4, which are 260 workgroups, 31); a wave's part is at least eight k16 groups.
    // Against the tiles at 32 rows: 12.8 and 13.6 us at 4096 x 4096, 23.4 and 26.2 at
    // 4096 x 16384; at 64 rows this form took 16.2 and 15.4, 31 and 28.
    s.rows = true;
    s.mb = 1;
    const int cts = (d_out + 63) / 64;
    s.splits = (int)std::max<long long>(1, std::min<long long>(kDnCUs / cts,
                                                               d / 16 / (8 * kDnWaves)));
    return s;
  }
  // Tile height and parts by an estimate of the time in us.  Its figures are fitted to
  // 711 timings, heights from 96 on and up to 16 parts of 22 shapes of 97 to 4768 rows and
  // 136 to 16384 columns, weights warm; its picks were at most 7 % behind the fastest
  // there, 4 % in 336 more of 6 shapes whose weights came from HBM, and in 714 of 16
  // shapes with and without GELU and residual 2 % on average, 14 % at most.  A step
  // costs a fixed 0.13 and per block of 32 rows 0.115 on an empty chip to 0.17 on a full
  // one (power; n tiles on the busiest CU, u the share of the others' work).  A tile's
  // start and end are hidden in part where two workgroups share a CU (MB <= 4);
  // above, 1.7 a block stands for 1.08 and an activation's or a residual's share.  Parts
  // are written, read and added.  Every row tile reads the weights, through the L2s at
  // 41 TB/s.
  s.rows = false;
  const long long nts = (d_out + kDnNT - 1) / kDnNT;
  const int steps = std::max(1, d / kDnStep);
  double best = 0.0;
  s.mb = 0;
  s.splits = 1;
  for (int mb = 8; mb >= 2; --mb) {
    const long long tiles = ((long long)M + 32 * mb - 1) / (32 * mb) * nts;
    // a part is at least eight steps
    const int most = std::max(1, std::min(16, steps / 8));
    for (int sp = 1; sp <= most; ++sp) {
      const double n = (double)((tiles * sp + kDnCUs - 1) / kDnCUs);
      const double u = (double)(tiles * sp) / (n * kDnCUs);
      double us = n * ((steps + sp - 1) / sp) * (0.127 + mb * (0.115 + 0.054 * u));
      us += mb <= 4 ? 4.06 + 1.08 * mb * (0.27 + 0.73 * n) : n * (4.06 + 1.7 * mb);
      if (sp > 1) us += 1.4 + (double)sp * M * d_out * 8.0 / 8.84e6;
      us += (double)((M + 32ll * mb - 1) / (32 * mb)) * d * d_out * 2.0 / 41e6;
      if (s.mb == 0 || us < best) {
        best = us;
        s.mb = mb;
        s.splits = sp;
      }
    }
  }
  return s;
}

// Workgroups of the layer's launch, and whether one grid dimension holds them.
static long long dense_items(int M, int d_out, const DenseShape& s) {
  const int width = s.rows ? 64 : kDnNT;
  return ((long long)M + 32 * s.mb - 1) / (32 * s.mb) * ((d_out + width - 1) / width) * s.splits;
}
bool dense_fits(int M, int d, int d_out) {
  return M <= 0 || dense_items(M, d_out, dense_shape(M, d, d_out)) <= (1 << 22);
}

size_t dense_scratch_bytes(int M, int d, int d_out) {
  if (M <= 0) return 0;
  const DenseShape s = dense_shape(M, d, d_out);
  return s.splits > 1 ? (size_t)s.splits * M * d_out * sizeof(float) : 0;
}

hipError_t launch_dense(const skip_problem_t& p, const void* rows, const int32_t* kept_offsets,
                        const int32_t* rows_idx, const void* packed, int d_out, const float* bias,
                        int act, const void* residual, const int32_t* residual_idx, void* Y,
                        int out_f32, void* scratch, hipStream_t st) {
  DenseArgs a;
  a.rows = static_cast<const bf16_t*>(rows);
  a.rows_idx = rows_idx;
  a.kept_offsets = kept_offsets;
  a.B = p.B;
  a.N = p.N;
  a.M = p.total_kept;
  a.d = p.d;
  a.d_out = d_out;
  a.Wp = static_cast<const u32x4*>(packed);
  a.bias = bias;
  a.residual = static_cast<const bf16_t*>(residual);
  a.residual_idx = residual_idx;
  a.act = act;
  a.out_f32 = out_f32;
  a.Y = Y;
  a.part = static_cast<float*>(scratch);
  if (a.M <= 0) return hipSuccess;
  const DenseShape s = dense_shape(a.M, a.d, d_out);
  a.splits = s.splits;
  a.n_items = (int)dense_items(a.M, d_out, s);
  const dim3 grid((unsigned)((a.n_items + 7) / 8 * 8));
#define SKIP_DENSE(MB) \
  hipLaunchKernelGGL(dense_tile_kernel<MB>, grid, dim3(kDnThreads), 0, st, a)
  if (s.rows) {
    hipLaunchKernelGGL(dense_rows_kernel, grid, dim3(64 * kDnWaves), 0, st, a);
  } else {
    switch (s.mb) {
      case 2: SKIP_DENSE(2); break;
      case 3: SKIP_DENSE(3); break;
      case 4: SKIP_DENSE(4); break;
      case 5: SKIP_DENSE(5); break;
      case 6: SKIP_DENSE(6); break;
      case 7: SKIP_DENSE(7); break;
      default: SKIP_DENSE(8); break;
    }
  }
#undef SKIP_DENSE
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const size_t n = (size_t)a.M * (d_out / 8);
  hipLaunchKernelGGL(dense_join_kernel, dim3((unsigned)std::min<size_t>((n + 255) / 256, 1 << 16)),
                     dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace skip
