// Passages held in 4 bits (the store that skip_bipartite_xattn_quant reads):
// writing them, reading them back, and their mean keys.
//
// A block of 32 values x is held as codes of {0, .5, 1, 1.5, 2, 3, 4, 6} with a
// sign and one power of two 2^(s - 127), the least with max|x| <= 7 * 2^(s - 127)
// (from there on 6 would be more than half a step away), s from 1 to 252: 4.25 bits a
// value, all of them finite (the largest is 6 * 2^125; infinities are held as it).  A
// key block is 32 features of one token, a value block 32 tokens of one feature,
// so that a lane of the attention's matrix products holds one block's values and
// one scale.  Store record (32 tokens, one head, d_h = D), 34 D bytes:
//   K        [t 2][chunk D/32][i 16][16 B]  token 16 t + i, features 32 chunk ..
//   V        [D][16 B]                      tokens 0 .. 31 of a feature
//   K scales [chunk % 2][i 16][t 2][chunk / 2]
//   V scales [feature % 32][feature / 32]
// the low nibble of a byte first.  One 4- or 2-byte load then gives a lane of the
// attention all its scales of a record.
//
// A wave makes one record at a time, through LDS of its own, so that it reads whole
// token rows and writes whole records.  160 passages of 256 tokens, 32 heads of 128 in
// bf16 (671 MB, 178 held): read in 140 us (6.05 TB/s, HBM); written in 200 to 230 (3.7
// to 4.2 TB/s), the waves waiting for 74 % of their time: 182 VGPRs leave two of them a
// SIMD, and each loads a record, codes it and stores it in turn.  The mean keys read the
// keys again, 61 us more (5.5 TB/s); a single passage has a workgroup for every 512
// columns only, and is bound by latency.
#include <algorithm>

#include "skip_common.h"
#include "skip_internal.h"
#include "skip_store.h"

namespace skip {

constexpr int kStoreWaves = 4;
constexpr int kStoreMaxGrid = 1 << 16;      // workgroups; the rest by stride

// Eight consecutive elements as floats.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    unpack8_bf16(*reinterpret_cast<const u32x4*>(p), x);
  } else {
    const float4 a = reinterpret_cast<const float4*>(p)[0];
    const float4 b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]),
                                         pack2_bf16(x[4], x[5]), pack2_bf16(x[6], x[7])};
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// Scale byte of a block whose largest magnitude has these bits (sign cleared).
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  const int s = (int)(amax >> 23) - 2 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)clampi(s, 1, 252);
}
// Eight values as codes (round to nearest even), the first in the low nibble.
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
  return r;
}
__device__ __forceinline__ void values8(uint32_t codes, float scale, float (&x)[8]) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
  const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
  const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
  const f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}

// First token of block i of the passage of tokens ts .. te - 1; false: the passage ends
// before it.  (The blocks go by the longest passage, and ts + 32 i of another one may
// pass 32 bits.)
__host__ __device__ bool store_block(int ts, int te, int i, int& t0) {
  if (i > (te - ts - 1) >> 5) return false;
  t0 = ts + 32 * i;
  return true;
}

// The work of a wave: record (passage j, block i of it, head h); false: none.
struct StoreItem {
  int h, t0, te;        // head, first token and end of the passage (source rows)
  size_t rec;           // record in the store
};
__device__ __forceinline__ bool store_item(const StoreShape& a, long long item, StoreItem& x) {
  const int hg = (int)(item % a.head_groups);
  const long long r = item / a.head_groups;
  const int i = (int)(r % a.blocks_max), j = (int)(r / a.blocks_max);
  int ts, te;
  range_of(a.passage_offsets, j, a.total_tokens, ts, te);
  x.h = hg * kStoreWaves + (int)(threadIdx.x >> 6);
  x.te = te;
  if (!store_block(ts, te, i, x.t0) || x.h >= a.heads) return false;
  const long long blk = (long long)a.passage_blocks[j] + i;
  if (blk < 0 || blk >= a.n_blocks) return false;      // outside the store: not touched
  x.rec = (size_t)blk * a.heads + x.h;
  return true;
}

template <typename T, int D>
__global__ void __launch_bounds__(64 * kStoreWaves)
store_write_kernel(StoreShape a, const T* __restrict__ Kh, const T* __restrict__ Vh,
                   uint8_t* __restrict__ data, long long items) {
  constexpr int C = D / 32, LPT = D / 8;      // chunks; lanes of a token row
  constexpr int TPL = 64 / LPT;               // token groups of a wave (4 or 8)
  constexpr int NT = 32 / TPL;                // tokens of a lane
  constexpr int REC = 34 * D;
  __shared__ __attribute__((aligned(16))) uint8_t buf[kStoreWaves][REC];
  const int lane = threadIdx.x & 63, f0 = 8 * (lane % LPT), g = lane / LPT;
  uint8_t* out = buf[threadIdx.x >> 6];
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    StoreItem x;
    if (!store_item(a, it, x)) continue;
    const size_t stride = (size_t)a.heads * D, base = (size_t)x.h * D + f0;
    // the lane's tokens: NT * g .. + NT - 1 of the block (past the passage: zeros)
    float v[NT][8], k[NT][8];
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      const int t = x.t0 + NT * g + q;
      const size_t off = (size_t)min(t, x.te - 1) * stride + base;
      load8(Kh + off, k[q]);
      load8(Vh + off, v[q]);
      if (t >= x.te)
#pragma unroll
        for (int e = 0; e < 8; ++e) k[q][e] = v[q][e] = 0.f;
    }
    // keys: four lanes share a block
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(k[q][e]) & 0x7fffffffu);
      m = max(m, (uint32_t)__shfl_xor((int)m, 1, kWave));
      m = max(m, (uint32_t)__shfl_xor((int)m, 2, kWave));
      const uint32_t s = scale_byte(m);
      const int t = NT * g + q, c = f0 / 32;
      *reinterpret_cast<uint32_t*>(out + (((t >> 4) * C + c) * 16 + (t & 15)) * 16 +
                                   ((f0 & 31) >> 1)) = codes8(k[q], __uint_as_float(s << 23));
      if ((lane & 3) == 0)
        out[32 * D + ((c & 1) * 16 + (t & 15)) * C + (t >> 4) * (C / 2) + (c >> 1)] = (uint8_t)s;
    }
    // values: the token groups of a feature share a block
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t m = 0;
#pragma unroll
      for (int q = 0; q < NT; ++q) m = max(m, __float_as_uint(v[q][e]) & 0x7fffffffu);
#pragma unroll
      for (int w = LPT; w < 64; w <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, w, kWave));
      const uint32_t s = scale_byte(m);
      const float sc = __uint_as_float(s << 23);
      uint32_t r = 0;
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0][e], v[1][e], sc, 0);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2][e], v[3][e], sc, 1);
      const int f = f0 + e;
      uint8_t* row = out + 16 * D + f * 16;
      if constexpr (NT == 8) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4][e], v[5][e], sc, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6][e], v[7][e], sc, 3);
        *reinterpret_cast<uint32_t*>(row + 4 * g) = r;
      } else {
        *reinterpret_cast<uint16_t*>(row + 2 * g) = (uint16_t)r;
      }
      if (g == 0) out[33 * D + (f & 31) * C + (f >> 5)] = (uint8_t)s;
    }
    // (the wave's own LDS, read in the order it was written)
    __builtin_amdgcn_wave_barrier();
    for (int u = lane; u < REC / 16; u += 64)
      reinterpret_cast<u32x4*>(data + x.rec * REC)[u] = reinterpret_cast<const u32x4*>(out)[u];
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(64 * kStoreWaves)
store_read_kernel(StoreShape a, const uint8_t* __restrict__ data, T* __restrict__ Kh,
                  T* __restrict__ Vh, long long items) {
  constexpr int C = D / 32, LPT = D / 8, TPL = 64 / LPT, NT = 32 / TPL, REC = 34 * D;
  __shared__ __attribute__((aligned(16))) uint8_t buf[kStoreWaves][REC];
  const int lane = threadIdx.x & 63, f0 = 8 * (lane % LPT), g = lane / LPT;
  uint8_t* in = buf[threadIdx.x >> 6];
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    StoreItem x;
    if (!store_item(a, it, x)) continue;
    for (int u = lane; u < REC / 16; u += 64)
      reinterpret_cast<u32x4*>(in)[u] = reinterpret_cast<const u32x4*>(data + x.rec * REC)[u];
    __builtin_amdgcn_wave_barrier();
    float v[8][8];                             // [feature][token of the lane]
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int f = f0 + e;
      const uint8_t* row = in + 16 * D + f * 16;
      const uint32_t codes = NT == 8 ? *reinterpret_cast<const uint32_t*>(row + 4 * g)
                                     : *reinterpret_cast<const uint16_t*>(row + 2 * g);
      values8(codes, __uint_as_float((uint32_t)in[33 * D + (f & 31) * C + (f >> 5)] << 23), v[e]);
    }
    const size_t stride = (size_t)a.heads * D, base = (size_t)x.h * D + f0;
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      const int t = NT * g + q, c = f0 / 32;
      if (x.t0 + t >= x.te) continue;          // rows behind the passage stay as they are
      const size_t off = (size_t)(x.t0 + t) * stride + base;
      const uint32_t codes = *reinterpret_cast<const uint32_t*>(
          in + (((t >> 4) * C + c) * 16 + (t & 15)) * 16 + ((f0 & 31) >> 1));
      const uint32_t s =
          in[32 * D + ((c & 1) * 16 + (t & 15)) * C + (t >> 4) * (C / 2) + (c >> 1)];
      float k[8], w[8];
      values8(codes, __uint_as_float(s << 23), k);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = v[e][q];
      store8(Kh + off, k);
      store8(Vh + off, w);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Mean key of every passage (float64 sums), each key head once per query head
// of its group: out [passages][heads * group * D].  Workgroup: 512 columns of a
// passage, its four waves every fourth token.
template <typename T>
__global__ void __launch_bounds__(256)
store_keys_kernel(const int32_t* __restrict__ passage_offsets, int total_tokens, int passages,
                  int width, int group, int d_h, const T* __restrict__ Kh,
                  float* __restrict__ out) {
  __shared__ double part[4][64][9];            // (9: spread over the banks)
  const int slices = (width + 511) / 512;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long it = blockIdx.x; it < (long long)passages * slices; it += gridDim.x) {
    const int j = (int)(it / slices), c = (int)(it % slices) * 512 + 8 * lane;
    int ts, te;
    range_of(passage_offsets, j, total_tokens, ts, te);
    double s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < width) {
      constexpr int U = 4;                     // rows in flight
      for (int t = ts + wave; t < te; t += 4 * U) {
        float x[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u)
          load8(Kh + (size_t)min(t + 4 * u, te - 1) * width + c, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (t + 4 * u < te)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += x[u][e];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[wave][lane][e] = s[e];
    __syncthreads();
    if (wave == 0 && c < width) {
      const double n = te > ts ? te - ts : 1;
      float* row = out + (size_t)j * width * group + (size_t)(c / d_h) * group * d_h + c % d_h;
      float m[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        m[e] = (float)((((part[0][lane][e] + part[1][lane][e]) + part[2][lane][e]) +
                        part[3][lane][e]) / n);
      for (int q = 0; q < group; ++q) store8(row + (size_t)q * d_h, m);
    }
    __syncthreads();
  }
}

static StoreShape shape_of(const skip_problem_t& p, const skip_kv_store_t& st,
                           const int32_t* passage_offsets, const int32_t* passage_blocks,
                           long long& items) {
  StoreShape a;
  a.passage_offsets = passage_offsets;
  a.passage_blocks = passage_blocks;
  a.total_tokens = p.total_tokens;
  a.n_blocks = st.n_blocks;
  a.heads = st.heads_kv;
  a.head_groups = (st.heads_kv + kStoreWaves - 1) / kStoreWaves;
  a.blocks_max = (p.L_max + 31) / 32;
  items = (long long)p.total_passages * a.blocks_max * a.head_groups;
  return a;
}

hipError_t launch_store_write(const skip_problem_t& p, const skip_kv_store_t& st, const void* Kh,
                              const void* Vh, const int32_t* passage_offsets,
                              const int32_t* passage_blocks, float* keys_out, hipStream_t s) {
  long long items;
  const StoreShape a = shape_of(p, st, passage_offsets, passage_blocks, items);
  if (items == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<long long>(items, kStoreMaxGrid));
  uint8_t* data = static_cast<uint8_t*>(st.data);
#define SKIP_STORE_WRITE(T, DD)                                                           \
  hipLaunchKernelGGL((store_write_kernel<T, DD>), grid, dim3(64 * kStoreWaves), 0, s, a,  \
                     (const T*)Kh, (const T*)Vh, data, items)
  if (p.dtype == SKIP_F32) {
    if (p.d_h == 64) SKIP_STORE_WRITE(float, 64);
    else SKIP_STORE_WRITE(float, 128);
  } else {
    if (p.d_h == 64) SKIP_STORE_WRITE(bf16_t, 64);
    else SKIP_STORE_WRITE(bf16_t, 128);
  }
#undef SKIP_STORE_WRITE
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !keys_out) return e;
  const int width = st.heads_kv * p.d_h;
  const long long n = (long long)p.total_passages * ((width + 511) / 512);
  const dim3 kgrid((unsigned)std::min<long long>(n, kStoreMaxGrid));
#define SKIP_STORE_KEYS(T)                                                                \
  hipLaunchKernelGGL((store_keys_kernel<T>), kgrid, dim3(256), 0, s, passage_offsets,     \
                     p.total_tokens, p.total_passages, width, p.H / st.heads_kv, p.d_h,   \
                     (const T*)Kh, keys_out)
  if (p.dtype == SKIP_F32) SKIP_STORE_KEYS(float);
  else SKIP_STORE_KEYS(bf16_t);
#undef SKIP_STORE_KEYS
  return hipGetLastError();
}

hipError_t launch_store_read(const skip_problem_t& p, const skip_kv_store_t& st,
                             const int32_t* passage_offsets, const int32_t* passage_blocks,
                             void* Kh, void* Vh, hipStream_t s) {
  long long items;
  const StoreShape a = shape_of(p, st, passage_offsets, passage_blocks, items);
  if (items == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<long long>(items, kStoreMaxGrid));
  const uint8_t* data = static_cast<const uint8_t*>(st.data);
#define SKIP_STORE_READ(T, DD)                                                            \
  hipLaunchKernelGGL((store_read_kernel<T, DD>), grid, dim3(64 * kStoreWaves), 0, s, a,   \
                     data, (T*)Kh, (T*)Vh, items)
  if (p.dtype == SKIP_F32) {
    if (p.d_h == 64) SKIP_STORE_READ(float, 64);
    else SKIP_STORE_READ(float, 128);
  } else {
    if (p.d_h == 64) SKIP_STORE_READ(bf16_t, 64);
    else SKIP_STORE_READ(bf16_t, 128);
  }
#undef SKIP_STORE_READ
  return hipGetLastError();
}

}  // namespace skip
