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
//   dense_rows_kernel : few rows: 32 MB rows x 64 columns, the contraction split
//                       over the workgroup's waves
//   dense_join_kernel : adds the parts of a contraction that several workgroups
//                       shared, in their order, and finishes
#include <algorithm>
#include <type_traits>

#include "skip_common.h"
#include "skip_internal.h"

namespace skip {

constexpr int kDnNT = 256;         // columns of a packed tile
constexpr int kDnKS = 32;          // contraction per step
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

// f(0), .., f(N-1) with compile-time indices.
template <int N, int I = 0, class F>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<N, I + 1>(f);
  }
}

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

__device__ __forceinline__ float dense_act(float x, int act) {
  switch (act) {
    case SKIP_ACT_RELU: return fmaxf(x, 0.f);
    // (erfc: 1 + erf would lose the tail below zero)
    case SKIP_ACT_GELU: return 0.5f * x * erfcf(x * -0.70710678118654752f);
    case SKIP_ACT_SILU: return x / (1.f + __expf(-x));
  }
  return x;
}

// Eight sums of row r, columns j .. j + 7: bias, activation, residual, store.
__device__ __forceinline__ void dense_finish8(const DenseArgs& a, int r, int j, float (&x)[8]) {
  if (a.bias) {
    const float4 b0 = reinterpret_cast<const float4*>(a.bias + j)[0];
    const float4 b1 = reinterpret_cast<const float4*>(a.bias + j)[1];
    x[0] += b0.x; x[1] += b0.y; x[2] += b0.z; x[3] += b0.w;
    x[4] += b1.x; x[5] += b1.y; x[6] += b1.z; x[7] += b1.w;
  }
  if (a.act != SKIP_ACT_NONE)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = dense_act(x[e], a.act);
  if (a.residual) {
    float y[8];
    unpack8_bf16(*reinterpret_cast<const u32x4*>(
                     a.residual + dense_row(a, a.residual_idx, r) * a.d_out + j), y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
  const size_t at = (size_t)r * a.d_out + j;
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

// Workgroup: 32 MB rows x 256 columns, a part of the contraction.  The row tile
// arrives in an LDS ring by direct global->LDS loads AH steps ahead and is
// published one step early; each wave's weights come from the packed copy into
// registers WD steps ahead, one coalesced run a load.  Items are dealt to the XCDs
// in runs, row tile fastest, so that the items of one XCD share their weights in
// its L2.
template <int MB>
__global__ void __launch_bounds__(kDnThreads, 1)
dense_tile_kernel(DenseArgs a) {
  constexpr int NB = 2;
  constexpr int RING = MB <= 6 ? 5 : 4, AH = RING - 1, WD = AH;
  constexpr int MT = 32 * MB, A_ELEMS = MT * kDnKS;
  constexpr int WCH = 32 * MB;                        // 16-byte chunks of a row tile per wave
  constexpr int NI = (WCH + 63) / 64;                 // direct loads they take
  constexpr int PITCH = 72;                           // floats of a row in the epilogue
  __shared__ __attribute__((aligned(1024))) union {
    bf16_t ring[RING * A_ELEMS];
    float out[4][32 * PITCH];
  } sh;
  static_assert(sizeof(sh.ring) <= 65536, "direct loads address 64 KiB of LDS");

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
  const int all_steps = a.d / kDnKS;
  const int s_begin = (int)((long long)all_steps * split / a.splits);
  const int ksteps = (int)((long long)all_steps * (split + 1) / a.splits) - s_begin;
  const int hh = lane >> 5, r32 = lane & 31;

  // the lane's 16-byte chunks of a row tile: chunk g is row g / 4, physical
  // chunk g % 4 holding logical chunk (g % 4) ^ (row / 2) % 4 (the operand
  // reads of 8 consecutive rows hit distinct banks)
  const bf16_t* asrc[NI];
#pragma unroll
  for (int q = 0; q < NI; ++q) {
    const int g = wave * WCH + min(q * 64 + lane, WCH - 1);
    const int trow = g >> 2;
    const int lc = (g & 3) ^ ((trow >> 1) & 3);
    asrc[q] = a.rows + dense_row(a, a.rows_idx, min(i0 + trow, a.M - 1)) * a.d +
              (size_t)s_begin * kDnKS + lc * 8;
  }
  const uint32_t ar_lds = lds_addr(sh.ring) + (uint32_t)(wave * WCH * 16);
  auto issue_a = [&](int s) {
#pragma unroll
    for (int q = 0; q < NI; ++q)
      if (q * 64 + lane < WCH)
        lds_dma16(asrc[q] + s * kDnKS,
                  __builtin_amdgcn_readfirstlane(
                      ar_lds + ((uint32_t)s % RING) * (A_ELEMS * 2) + q * 1024));
  };
  const u32x4* wsrc = a.Wp + ((size_t)(nt * 8 + wave * NB) * all_steps + s_begin) * 128 + lane;
  const size_t wblk = (size_t)all_steps * 128;        // from one 32-column block to the next
  auto load_w = [&](int s, int kk, u32x4 (&w)[NB]) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) w[nb] = wsrc[nb * wblk + (size_t)s * 128 + kk * 64];
  };

  f32x16_t acc[NB][MB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[nb][mb][v] = 0.f;

  int aoff[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk)
    aoff[kk] = r32 * kDnKS + (((2 * kk + hh) ^ ((r32 >> 1) & 3)) << 3);
  auto read_a = [&](int s, int kk, u32x4 (&x)[MB]) {
    const bf16_t* At = sh.ring + ((uint32_t)s % RING) * A_ELEMS + aoff[kk];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
      x[mb] = *reinterpret_cast<const u32x4*>(At + mb * 32 * kDnKS);
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

#pragma unroll
  for (int q = 0; q < AH; ++q)
    if (q < ksteps) issue_a(q);
  u32x4 w[WD][2][NB];
#pragma unroll
  for (int t = 0; t < WD; ++t)
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) load_w(min(t, ksteps - 1), kk, w[t][kk]);
  wait_vmcnt<0>();
  barrier_nofence();
  u32x4 f0[MB], f1[MB];
  read_a(0, 0, f0);

  // Step s: wait for this wave's part of the row tile of step s+1 (issued
  // after it: the weights of AH - 1 steps and, while they exist, the tiles of
  // steps s+2 .. s+AH-1), barrier (publishes that tile; the slot of step s-1
  // is free), request the tile of step s+AH, multiply step s and read the
  // first operands of step s+1 (past the last step: stale values that nothing
  // uses).  The tail steps (after the last whole group of WD; every tile is
  // requested by then) load nothing and wait for all.
  static_assert(AH >= WD && AH < RING, "tail steps request no tile; a slot is free");
  constexpr int WQ = (AH - 1) * 2 * NB;
  auto step = [&](int s, u32x4 (&ws)[2][NB], auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    if (TAIL) wait_vmcnt<0>();
    else if (s + AH <= ksteps) wait_vmcnt<WQ + (AH - 2) * NI>();
    else wait_vmcnt<WQ>();
    barrier_nofence();
    if (!TAIL && s + AH < ksteps) issue_a(s + AH);
    __builtin_amdgcn_sched_barrier(0);
    read_a(s, 1, f1);
    multiply(f0, ws[0]);
    // unconditional (the last steps reload the final fragments): a
    // conditional load would make the compiler drain the queue before the
    // next use of w
    if (!TAIL) load_w(min(s + WD, ksteps - 1), 0, ws[0]);
    __builtin_amdgcn_sched_barrier(0);
    read_a(s + 1, 0, f0);
    multiply(f1, ws[1]);
    if (!TAIL) load_w(min(s + WD, ksteps - 1), 1, ws[1]);
    __builtin_amdgcn_sched_barrier(0);
  };
  int s = 0;
  for (; s + WD <= ksteps; s += WD) {
#pragma unroll
    for (int t = 0; t < WD; ++t) step(s + t, w[t], std::false_type{});
  }
#pragma unroll
  for (int t = 0; t < WD - 1; ++t)
    if (s + t < ksteps) step(s + t, w[t], std::true_type{});

  // Accumulator element v of block (nb, mb) is row mb*32 + 8*(v/4) + 4*hh + v%4,
  // column 64*wave + 32*nb + r32: through the wave's own LDS, 32 rows at a time,
  // so that a lane finishes eight columns of a row
  __syncthreads();                                    // the ring is read
  float* out = sh.out[wave];
  unrolled<MB>([&](auto mb_) {
    constexpr int mb = decltype(mb_)::value;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        out[(8 * (v >> 2) + 4 * hh + (v & 3)) * PITCH + 32 * nb + r32] = acc[nb][mb][v];
    __builtin_amdgcn_wave_barrier();
    for (int q = 0; q < 4; ++q) {
      const int lr = 8 * q + (lane >> 3), r = i0 + mb * 32 + lr;
      const int j = j0 + 64 * wave + 8 * (lane & 7);
      float x[8];
      *reinterpret_cast<float4*>(x) =
          *reinterpret_cast<const float4*>(out + lr * PITCH + 8 * (lane & 7));
      *reinterpret_cast<float4*>(x + 4) =
          *reinterpret_cast<const float4*>(out + lr * PITCH + 8 * (lane & 7) + 4);
      if (r < a.M && j < a.d_out) {
        if (a.splits > 1) dense_part8(a, split, r, j, x);
        else dense_finish8(a, r, j, x);
      }
    }
    __builtin_amdgcn_wave_barrier();
  });
}

// Few rows: bound by the weights' way from memory, so every wave streams its own
// part of them (64 columns, an eighth of the workgroup's contraction) straight
// into registers, a batch of loads ahead of the products; the rows come from the
// L2.  The waves' sums meet in LDS, added in wave order.
template <int MB>
__global__ void __launch_bounds__(64 * kDnWaves, 2)
dense_rows_kernel(DenseArgs a) {
  constexpr int NB = 2, U = MB == 1 ? 4 : 2;          // k16 groups a batch
  __shared__ float red[kDnWaves][16][64];
  const int per_xcd = gridDim.x / 8;
  int item = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (item >= a.n_items) return;
  const int MTL = (a.M + 32 * MB - 1) / (32 * MB);
  const int mt = item % MTL;
  item /= MTL;
  const int split = item % a.splits, ct = item / a.splits;
  const int i0 = mt * 32 * MB, j0 = ct * 64;
  const int lane = threadIdx.x & 63, hh = lane >> 5, r32 = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.d / 16, parts = a.splits * kDnWaves, me = split * kDnWaves + wv;
  const int g0 = (int)((long long)me * G / parts), g1 = (int)((long long)(me + 1) * G / parts);
  const int gl = max(g1 - 1, 0);

  const bf16_t* ap[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
    ap[mb] = a.rows + dense_row(a, a.rows_idx, min(i0 + mb * 32 + r32, a.M - 1)) * a.d + hh * 8;
  const u32x4* wp = a.Wp + (size_t)ct * 2 * G * 64 + lane;
  struct Batch {
    u32x4 x[U][MB], w[U][NB];
  };
  auto load = [&](Batch& b, int g) {                  // groups past the wave's are not multiplied
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t gg = (size_t)min(g + u, gl);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) b.w[u][nb] = wp[((size_t)nb * G + gg) * 64];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
        b.x[u][mb] = *reinterpret_cast<const u32x4*>(ap[mb] + gg * 16);
    }
  };
  f32x16_t acc[NB][MB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[nb][mb][v] = 0.f;
  auto multiply = [&](const Batch& b, int g) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g + u < g1)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            acc[nb][mb] = mfma32_bf16(b.x[u][mb], b.w[u][nb], acc[nb][mb]);
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
  // after the other: thread (row 32 in eight, four columns) of the first 256
  // adds the waves' sums of eight columns
  unrolled<MB * NB>([&](auto i_) {
    constexpr int mb = decltype(i_)::value / NB, nb = decltype(i_)::value % NB;
      if (mb + nb > 0) __syncthreads();
#pragma unroll
      for (int v = 0; v < 16; ++v) red[wv][v][lane] = acc[nb][mb][v];
      __syncthreads();
      if (threadIdx.x < 128) {
        const int lr = threadIdx.x >> 2, c8 = (threadIdx.x & 3) * 8;
        const int v = 4 * (lr >> 3) + (lr & 3), l = 32 * ((lr >> 2) & 1) + c8;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = red[0][v][l + e];
#pragma unroll
          for (int u = 1; u < kDnWaves; ++u) x[e] += red[u][v][l + e];
        }
        const int r = i0 + mb * 32 + lr, j = j0 + nb * 32 + c8;
        if (r < a.M && j < a.d_out) {
          if (a.splits > 1) dense_part8(a, split, r, j, x);
          else dense_finish8(a, r, j, x);
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
    dense_finish8(a, r, j, x);
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
  if (M <= 96) {
    s.rows = true;
    s.mb = (M + 31) / 32;
    const int cts = (d_out + 63) / 64;
    // a wave's part is at least eight k16 groups
    s.splits = (int)std::max<long long>(1, std::min<long long>((kDnCUs + cts - 1) / cts,
                                                               d / 16 / (8 * kDnWaves)));
    return s;
  }
  s.rows = false;
  const long long nts = (d_out + kDnNT - 1) / kDnNT;
  // rounds of workgroups times their rows, over tile heights
  long long best = -1;
  s.mb = 8;
  s.splits = 1;
  for (int mb = 8; mb >= 3; --mb) {
    const long long tiles = (M + 32 * mb - 1) / (32 * mb) * nts;
    // a part is at least 16 steps
    const int most = std::max(1, std::min(16, d / kDnKS / 16));
    for (int sp = 1; sp <= most; ++sp) {
      const long long rounds = (tiles * sp + kDnCUs - 1) / kDnCUs;
      const long long cost = (rounds * (mb * 64 + 32) * 1024) / sp + (sp > 1 ? 4096 * sp : 0);
      if (best < 0 || cost < best) {
        best = cost;
        s.mb = mb;
        s.splits = sp;
      }
    }
  }
  return s;
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
  const int width = s.rows ? 64 : kDnNT;
  const long long items = (long long)((a.M + 32 * s.mb - 1) / (32 * s.mb)) *
                          ((d_out + width - 1) / width) * s.splits;
  if (items > (1 << 22)) return hipErrorInvalidValue;
  a.n_items = (int)items;
  const dim3 grid((unsigned)((items + 7) / 8 * 8));
#define SKIP_DENSE(K, MB, T) hipLaunchKernelGGL((K<MB>), grid, dim3(T), 0, st, a)
  if (s.rows) {
    switch (s.mb) {
      case 1: SKIP_DENSE(dense_rows_kernel, 1, 64 * kDnWaves); break;
      case 2: SKIP_DENSE(dense_rows_kernel, 2, 64 * kDnWaves); break;
      default: SKIP_DENSE(dense_rows_kernel, 3, 64 * kDnWaves); break;
    }
  } else {
    switch (s.mb) {
      case 3: SKIP_DENSE(dense_tile_kernel, 3, kDnThreads); break;
      case 4: SKIP_DENSE(dense_tile_kernel, 4, kDnThreads); break;
      case 5: SKIP_DENSE(dense_tile_kernel, 5, kDnThreads); break;
      case 6: SKIP_DENSE(dense_tile_kernel, 6, kDnThreads); break;
      case 7: SKIP_DENSE(dense_tile_kernel, 7, kDnThreads); break;
      default: SKIP_DENSE(dense_tile_kernel, 8, kDnThreads); break;
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
