// Sparse cross-attention over passages held in 4 bits (paper App. B.3, Def. B.3
// attention rule; the store's format is at the top of store.hip).
//
// For kept row i of question b and query head h, with key head h / G,
//   e_m = sm_scale * <Q[i,h], K[m,h/G]>,  O = softmax(e) . V,  LSE = log sum exp e
// over the tokens m of the passages adjacent to i.
//
// A (row, query head of the group) pair is one virtual row: row v of an item is
// kept row v / G and query head v % G, and all of them meet the same keys.  A
// workgroup takes one (question, key head) and up to ROWS virtual rows.  Its work
// is a list of units, (passage, segment of its tokens, 32 of the rows adjacent
// to it), in the order of passages and segments, which its waves take one after
// the other.  A wave computes its unit alone, 64 tokens (two records) at a time,
// with no LDS and no barrier: the store holds each operand of
//   S^T (64 tokens x 32 rows) = K . Q^T,  O^T (D x 32 rows) += V^T . P^T
// (v_mfma_f32_32x32x16_bf16) as its lane takes it, 16 bytes and one scale a
// block, which the lane turns into bf16 exactly (a 2-bit significand times a
// power of two).  Which feature or token a contraction slot stands for is free as
// long as both operands agree, so the softmax weights stay in the lanes that
// computed them, too: lane l (n = l % 32, hh = l / 32) holds row n's logits of
// tokens 32 hh + 16 t + i in element i of product t.  The online softmax is in
// base 2 and float32; a weight enters the second product as a sum of bf16 pieces
// (two for bf16 output, 2^-16 relative; three for float output, 2^-24).
//
// A unit's (O, max, sum) is merged into the item's, float32 in LDS, in the order
// of the list, so that the result does not depend on which wave was faster: a
// wave waits until every unit of earlier passages and segments is merged.  (Units
// are taken in order, so the earliest one that is not merged never waits.)
#include <algorithm>
#include <type_traits>

#include "skip_common.h"
#include "skip_internal.h"
#include "skip_store.h"

namespace skip {

constexpr float kQLog2e = 1.4426950408889634f;
constexpr float kQLn2 = 0.6931471805599453f;
constexpr float kQLazy = 8.f;              // log2 slack of the softmax reference maximum
constexpr int kQWaves = 8;
constexpr int kQThreads = 64 * kQWaves;
constexpr int kQMaxP = 64;                 // passages of a question

// Value of lane l ^ 32.
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x),
                                                  false, false);
  return __uint_as_float(__lane_id() < 32 ? r[1] : r[0]);
}

// Position of the n-th (from 0) set bit of x; n < popcount(x).
__device__ __forceinline__ int nth_set(uint64_t x, int n) {
  int pos = 0;
#pragma unroll
  for (int w = 32; w >= 1; w >>= 1) {
    const int c = __popcll(x & ((1ull << w) - 1ull));
    if (n >= c) {
      n -= c;
      x >>= w;
      pos += w;
    }
  }
  return pos;
}

// Eight 4-bit values (a dword) as bf16, exactly, times 2^(byte B of scales - 127).
template <int B>
__device__ __forceinline__ float scale_of(uint32_t scales) {
  return __uint_as_float(((scales >> (8 * B)) & 0xffu) << 23);
}
__device__ __forceinline__ u32x4 expand8(uint32_t codes, float scale) {
  return u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// One addition to an LDS counter for the whole wave; returns the value before it,
// uniform.  The wave barriers keep the branch on lane 0 to itself: without them
// the compiler joins it with the next one like it across a loop's back edge, and
// the other lanes run ahead.
__device__ __forceinline__ int wave_fetch_add(int* counter) {
  __builtin_amdgcn_wave_barrier();
  int x = 0;
  if (__lane_id() == 0) x = atomicAdd(counter, 1);
  __builtin_amdgcn_wave_barrier();
  return __builtin_amdgcn_readfirstlane(x);
}

template <int N, int I = 0, class F>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<N, I + 1>(f);
  }
}

struct QuantAttnArgs {
  const bf16_t* q;                  // kept rows, or V where kept_idx is given
  const int32_t* kept_idx;
  const int32_t* kept_offsets;
  const int32_t* query_passages;
  const int32_t* passage_offsets;
  const int32_t* passage_blocks;
  const uint64_t* rowmask;
  const uint8_t* store;
  void* O;
  float* lse;
  float* part;                      // partials of split items
  long long n_blocks;
  int N, H, heads_kv, G, groups, chunks, splits, rows_chunk;   // rows_chunk: kept rows an item
  int total_kept, total_passages, total_tokens, k_max, P_max, o_f32;
  float scale_log2;
};

// Floats of one split's partial of an item: rows of D values, maxima, sums.
__device__ __host__ __forceinline__ size_t part_floats(int rows, int D) {
  return ((size_t)rows * (D + 2) + 3) / 4 * 4;
}

// What a workgroup works on.
struct QuantItem {
  int b, hk, chunk, split;
  int k0, i0, nk;                   // the question's first kept row; the item's rows i0 .. + nk - 1
  int p0, P;
};
// Chunks and splits of a (question, key head) follow one another on one XCD
// (workgroup id L goes to XCD L % 8), whose L2 then holds its passages once.
__device__ __forceinline__ bool quant_item(const QuantAttnArgs& a, int L, QuantItem& x) {
  const int per = a.chunks * a.splits;
  const int grp = (L & 7) + 8 * ((L >> 3) / per);
  if (grp >= a.groups) return false;
  const int sub = (L >> 3) % per;
  x.chunk = sub / a.splits;
  x.split = sub % a.splits;
  x.b = grp / a.heads_kv;
  x.hk = grp % a.heads_kv;
  int k1, p1;
  range_of(a.kept_offsets, x.b, a.total_kept, x.k0, k1);
  range_of(a.query_passages, x.b, a.total_passages, x.p0, p1);
  const int kq = min(k1 - x.k0, a.k_max);
  x.P = min(min(p1 - x.p0, a.P_max), kQMaxP);
  const int nch = (kq + a.rows_chunk - 1) / a.rows_chunk;
  if (x.chunk >= nch) return false;
  const int rpc = (kq + nch - 1) / nch;                 // rows spread evenly over the chunks
  x.i0 = x.chunk * rpc;
  x.nk = min(kq, x.i0 + rpc) - x.i0;
  return x.nk > 0;
}

template <int D, int ROWS, int PIECES>
__global__ void __launch_bounds__(kQThreads, 2)
attn_quant_kernel(QuantAttnArgs a) {
  constexpr int C = D / 32, KH = D / 64;    // feature chunks of a record; pairs of them
  constexpr int FB = D / 32;                // 32-feature blocks of O
  constexpr int REC = kStoreRecord<D>;
  constexpr int NC4 = D / 4;                // 4-float chunks of an accumulator row
  constexpr int MW = (ROWS + 63) / 64;      // words of a row mask
  __shared__ __attribute__((aligned(16))) float Oacc[ROWS * D];
  __shared__ float m_acc[ROWS], l_acc[ROWS];
  __shared__ uint64_t rmask[MW][kQMaxP];    // virtual rows adjacent to each passage
  __shared__ int p_len[kQMaxP], p_blk[kQMaxP], p_cnt[kQMaxP], u_first[kQMaxP];
  __shared__ int u_total, seg_tiles, next_unit, merged;

  QuantItem it;
  if (!quant_item(a, blockIdx.x, it)) return;
  const int G = a.G, nv = it.nk * G, P = it.P;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;

  // accumulators, passages, adjacent rows of each
  for (int i = tid; i < nv * NC4; i += kQThreads)
    reinterpret_cast<float4*>(Oacc)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = tid; i < nv; i += kQThreads) {
    m_acc[i] = -INFINITY;
    l_acc[i] = 0.f;
  }
  if (tid < P) {
    int ts, te;
    range_of(a.passage_offsets, it.p0 + tid, a.total_tokens, ts, te);
    p_len[tid] = te - ts;
    p_blk[tid] = a.passage_blocks[it.p0 + tid];
  }
  if (wave < MW) {
    const uint64_t mk = tid < nv ? a.rowmask[it.k0 + it.i0 + tid / G] : 0ull;
    for (int j = 0; j < P; ++j) {
      const uint64_t bal = __ballot((mk >> j) & 1ull);
      if (lane == 0) rmask[wave][j] = bal;
    }
  }
  __syncthreads();
  // the list of units: 32-row blocks of every adjacent passage, each over
  // segments of seg_tiles tiles
  if (wave == 0) {
    int cnt = 0, tiles = 0;
    if (lane < P) {
#pragma unroll
      for (int w = 0; w < MW; ++w) cnt += __popcll(rmask[w][lane]);
      tiles = (p_len[lane] + 63) / 64;
    }
    const int nblk = tiles > 0 ? (cnt + 31) / 32 : 0;
    int work = nblk * tiles;
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) work += __shfl_xor(work, s, kWave);
    // about four units a wave, two tiles at least
    const int st = max(2, work / (4 * kQWaves * a.splits));
    const int units = nblk * ((tiles + st - 1) / st);
    int x = units;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int y = __shfl_up(x, s, kWave);
      if (lane >= s) x += y;
    }
    if (lane < P) {
      p_cnt[lane] = cnt;
      u_first[lane] = x - units;
    }
    if (lane == kWave - 1) {
      const int first = (int)((long long)x * it.split / a.splits);
      u_total = (int)((long long)x * (it.split + 1) / a.splits);
      next_unit = first;
      merged = first;
      seg_tiles = st;
    }
  }
  __syncthreads();
  const int U = u_total, st = seg_tiles, u_begin = merged;
  const int my_first = lane < P ? u_first[lane] : 0x7fffffff;
  __syncthreads();                           // every wave has read `merged`

  const uint32_t neg = (a.scale_log2 < 0.f) ? 0x80008000u : 0u;   // folded into the queries
  // (not zero: masked logits stay -inf)
  const float sc = fmaxf(fabsf(a.scale_log2), 1e-30f);
  const int ki = 4 * (n >> 3) + (n & 3), kb = (n >> 2) & 1;       // the lane's key row

  for (;;) {
    const int u = wave_fetch_add(&next_unit);
    if (u >= U) break;
    // passage of the unit (the last one that starts at or before it; empty
    // passages start where the next does)
    const int j = __popcll(__ballot(my_first <= u)) - 1;
    const int cnt = __builtin_amdgcn_readfirstlane(p_cnt[j]);
    const int len = __builtin_amdgcn_readfirstlane(p_len[j]);
    const int blk0 = __builtin_amdgcn_readfirstlane(p_blk[j]);
    const int uf = __builtin_amdgcn_readfirstlane(u_first[j]);
    const int nblk = (cnt + 31) / 32;
    const int seg = (u - uf) / nblk, rb = (u - uf) % nblk;
    const int t0 = seg * st * 64, t1 = min(len, t0 + st * 64);
    const int last_blk = (len - 1) >> 5;

    // this lane's row (past the block's rows: a placeholder that is not merged)
    int row = -1;
    {
      int m = 32 * rb + n;
      if (m < cnt) {
#pragma unroll
        for (int w = 0; w < MW; ++w) {
          const uint64_t bits = rmask[w][j];
          const int c = __popcll(bits);
          if (row < 0 && m < c) row = 64 * w + nth_set(bits, m);
          m -= c;
        }
      }
    }
    u32x4 qf[4 * KH];                        // features 64 kh + 32 hh .. + 31
    {
      const int v = max(row, 0);
      const int kr = it.k0 + it.i0 + v / G;
      const size_t r = a.kept_idx
          ? (size_t)it.b * a.N + clampi(a.kept_idx[kr], 0, a.N - 1) : (size_t)kr;
      const bf16_t* src = a.q + (r * a.H + (size_t)(it.hk * G + v % G)) * D + 32 * hh;
#pragma unroll
      for (int kh = 0; kh < KH; ++kh)
#pragma unroll
        for (int s = 0; s < 4; ++s)
          qf[4 * kh + s] = *reinterpret_cast<const u32x4*>(src + 64 * kh + 8 * s) ^ neg;
    }

    // record of the passage's block i (past its last block: that one, masked)
    auto record = [&](int i) -> const uint8_t* {
      long long blk = (long long)blk0 + min(i, last_blk);
      blk = blk < 0 ? 0 : (blk >= a.n_blocks ? a.n_blocks - 1 : blk);
      return a.store + ((size_t)blk * a.heads_kv + it.hk) * REC;
    };
    u32x4 kx[2][KH], vx[FB];
    uint32_t ks = 0, vs = 0;
    auto load_k = [&](int t) {
      const uint8_t* rec = record((t >> 5) + kb);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int kh = 0; kh < KH; ++kh)
          kx[h][kh] = *reinterpret_cast<const u32x4*>(rec + ((h * C + 2 * kh + hh) * 16 + ki) * 16);
      const uint8_t* sp = rec + 32 * D + (hh * 16 + ki) * C;
      ks = C == 4 ? *reinterpret_cast<const uint32_t*>(sp) : *reinterpret_cast<const uint16_t*>(sp);
    };
    auto load_v = [&](int t) {
      const uint8_t* rec = record((t >> 5) + hh);
#pragma unroll
      for (int fb = 0; fb < FB; ++fb)
        vx[fb] = *reinterpret_cast<const u32x4*>(rec + 16 * D + (32 * fb + n) * 16);
      const uint8_t* sp = rec + 33 * D + n * C;
      vs = C == 4 ? *reinterpret_cast<const uint32_t*>(sp) : *reinterpret_cast<const uint16_t*>(sp);
    };

    f32x16_t acc[FB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[fb][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    load_k(t0);
    load_v(t0);
    for (int t = t0; t < t1; t += 64) {
      f32x16_t s[2];
      unrolled<2>([&](auto h_) {
        constexpr int h = decltype(h_)::value;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[h][i] = 0.f;
        unrolled<KH>([&](auto kh_) {
          constexpr int kh = decltype(kh_)::value;
          const float scl = scale_of<h * KH + kh>(ks);
#pragma unroll
          for (int q = 0; q < 4; ++q)
            s[h] = mfma32_bf16(expand8(kx[h][kh][q], scl), qf[4 * kh + q], s[h]);
        });
      });
      // the next tile's keys land during the softmax and the second product
      // (past the segment: the last tile again, unused)
      const int tn = min(t + 64, (t1 - 1) & ~63);
      load_k(tn);
      if (t + 64 > t1) {
        const int rem = t1 - t - 32 * hh;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (16 * h + i >= rem) s[h][i] = -INFINITY;
      }
      float lm = s[0][0];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) lm = fmaxf(lm, s[h][i]);
      // the reference maximum moves when a logit exceeds it by more than kQLazy
      // (weights stay <= 2^kQLazy), so most tiles need no exchange or rescale
      if (__any(lm * sc > m_run + kQLazy)) {
        const float mx = fmaxf(lm, other_half(lm)) * sc;
        if (mx > m_run + kQLazy) {
          const float alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - mx);
          m_run = mx;
          l_run *= alpha;
#pragma unroll
          for (int fb = 0; fb < FB; ++fb) acc[fb] *= alpha;
        }
      }
      // (a segment's first tile has a token in every column, so m_run is finite)
      float ls = 0.f;
      unrolled<4>([&](auto q_) {
        constexpr int q = decltype(q_)::value, h = q >> 1, i0 = 8 * (q & 1);
        u32x4 pc[PIECES];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float p0 = __builtin_amdgcn_exp2f(fmaf(s[h][i0 + 2 * e], sc, -m_run));
          float p1 = __builtin_amdgcn_exp2f(fmaf(s[h][i0 + 2 * e + 1], sc, -m_run));
          ls += p0 + p1;
          // all pieces but the last are truncated, the rest is exact
#pragma unroll
          for (int c = 0; c + 1 < PIECES; ++c) {
            const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
            pc[c][e] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
            p0 -= __uint_as_float(b0 & 0xffff0000u);
            p1 -= __uint_as_float(b1 & 0xffff0000u);
          }
          pc[PIECES - 1][e] = pack2_bf16(p0, p1);
        }
        unrolled<FB>([&](auto fb_) {
          constexpr int fb = decltype(fb_)::value;
          const u32x4 va = expand8(vx[fb][q], scale_of<fb>(vs));
#pragma unroll
          for (int c = 0; c < PIECES; ++c) acc[fb] = mfma32_bf16(va, pc[c], acc[fb]);
        });
      });
      l_run += ls;
      load_v(tn);
    }

    // merge in the order of the list: every unit of earlier passages and
    // segments first (the others of this one have other rows)
    const int before = max(uf + seg * nblk, u_begin);
    while (__hip_atomic_load(&merged, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) < before)
      __builtin_amdgcn_s_sleep(1);
    asm volatile("" ::: "memory");
    const float l_tot = l_run + other_half(l_run);
    if (row >= 0) {
      const float mo = m_acc[row], lo = l_acc[row];
      const float mn = fmaxf(mo, m_run);
      const float fa = __builtin_amdgcn_exp2f(mo - mn);     // 0 while the row is empty
      const float fc = __builtin_amdgcn_exp2f(m_run - mn);
      float4* orow = reinterpret_cast<float4*>(Oacc + row * D);
#pragma unroll
      for (int fb = 0; fb < FB; ++fb)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          // features 32 fb + 8 c + 4 hh .. + 3
          float4& o = orow[(8 * fb + 2 * c + hh) ^ (row & (NC4 - 1))];
          o = make_float4(fmaf(o.x, fa, acc[fb][4 * c] * fc), fmaf(o.y, fa, acc[fb][4 * c + 1] * fc),
                          fmaf(o.z, fa, acc[fb][4 * c + 2] * fc),
                          fmaf(o.w, fa, acc[fb][4 * c + 3] * fc));
        }
      if (hh == 0) {
        m_acc[row] = mn;
        l_acc[row] = fmaf(lo, fa, l_tot * fc);
      }
    }
    wait_lgkm0();
    wave_fetch_add(&merged);
  }
  __syncthreads();

  if (a.splits > 1) {
    // this split's partial: rows of D values, then maxima and sums
    float* po = a.part + ((size_t)((it.b * a.heads_kv + it.hk) * a.chunks + it.chunk) * a.splits +
                          it.split) * part_floats(a.rows_chunk * G, D);
    for (int e = tid; e < nv * NC4; e += kQThreads) {
      const int ri = e / NC4, q = e % NC4;
      reinterpret_cast<float4*>(po)[e] =
          reinterpret_cast<const float4*>(Oacc + ri * D)[q ^ (ri & (NC4 - 1))];
    }
    float* pm = po + (size_t)(a.rows_chunk * G) * D;
    for (int i = tid; i < nv; i += kQThreads) {
      pm[i] = m_acc[i];
      pm[a.rows_chunk * G + i] = l_acc[i];
    }
    return;
  }
  // O = acc / sum for every row, and the LSE (0 and -inf without neighbours)
  for (int e = tid; e < nv * NC4; e += kQThreads) {
    const int ri = e / NC4, q = e % NC4;
    const float4 v = reinterpret_cast<const float4*>(Oacc + ri * D)[q ^ (ri & (NC4 - 1))];
    const float l = l_acc[ri];
    const float inv = (l > 0.f) ? 1.f / l : 0.f;
    const size_t off = ((size_t)(it.k0 + it.i0 + ri / G) * a.H + it.hk * G + ri % G) * D + q * 4;
    if (a.o_f32)
      *reinterpret_cast<float4*>(static_cast<float*>(a.O) + off) =
          make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    else
      *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.O) + off) =
          make_uint2(pack2_bf16(v.x * inv, v.y * inv), pack2_bf16(v.z * inv, v.w * inv));
  }
  if (a.lse)
    for (int i = tid; i < nv; i += kQThreads) {
      const float l = l_acc[i];
      a.lse[(size_t)(it.k0 + it.i0 + i / G) * a.H + it.hk * G + i % G] =
          (l > 0.f) ? (m_acc[i] + log2f(l)) * kQLn2 : -INFINITY;
    }
}

// The splits' partials of each item, added in their order.
template <int D>
__global__ void __launch_bounds__(256)
attn_quant_merge_kernel(QuantAttnArgs a) {
  constexpr int NC4 = D / 4;
  // one (group, chunk) a workgroup
  const int grp = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  QuantItem it;
  const int L = (grp & 7) + 8 * ((grp >> 3) * a.chunks * a.splits + chunk * a.splits);
  if (!quant_item(a, L, it)) return;
  const int G = a.G, nv = it.nk * G, S = a.splits;
  const size_t rows = (size_t)a.rows_chunk * G, step = part_floats(a.rows_chunk * G, D);
  const float* po = a.part + (size_t)((it.b * a.heads_kv + it.hk) * a.chunks + chunk) * S * step;
  const float* pm = po + rows * D;
  const float* pl = pm + rows;
  for (int e = threadIdx.x; e < nv * NC4; e += 256) {
    const int ri = e / NC4, q = e % NC4;
    float M = -INFINITY;
    for (int s = 0; s < S; ++s) M = fmaxf(M, pm[s * step + ri]);
    const float ref = M == -INFINITY ? 0.f : M;
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < S; ++s) {
      const float f = __builtin_amdgcn_exp2f(pm[s * step + ri] - ref);
      l = fmaf(pl[s * step + ri], f, l);
      const float4 x = reinterpret_cast<const float4*>(po + s * step)[e];
      o.x = fmaf(x.x, f, o.x);
      o.y = fmaf(x.y, f, o.y);
      o.z = fmaf(x.z, f, o.z);
      o.w = fmaf(x.w, f, o.w);
    }
    const float inv = (l > 0.f) ? 1.f / l : 0.f;
    const size_t at = (size_t)(it.k0 + it.i0 + ri / G) * a.H + it.hk * G + ri % G;
    if (a.o_f32)
      *reinterpret_cast<float4*>(static_cast<float*>(a.O) + at * D + q * 4) =
          make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    else
      *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.O) + at * D + q * 4) =
          make_uint2(pack2_bf16(o.x * inv, o.y * inv), pack2_bf16(o.z * inv, o.w * inv));
    if (a.lse && q == 0) a.lse[at] = (l > 0.f) ? (M + log2f(l)) * kQLn2 : -INFINITY;
  }
}

// How a problem is cut: virtual rows of an item, chunks of a question, splits of
// an item's list.
struct QuantShape {
  int rows, chunks, rows_chunk, splits;
};
static QuantShape quant_shape(const skip_problem_t& p, int heads_kv) {
  const int G = p.H / heads_kv;
  const long long groups = (long long)p.B * heads_kv;
  QuantShape s;
  for (int rows : {192, 64, 32}) {
    s.rows = rows;
    s.rows_chunk = std::max(1, rows / G);
    s.chunks = (p.k_max + s.rows_chunk - 1) / s.rows_chunk;
    if (groups * s.chunks >= 512) break;
  }
  s.splits = 1;
  const long long wgs = groups * s.chunks;
  if (wgs > 0 && wgs < 256) {
    // at least eight tiles of 64 tokens a split
    const long long tiles = (long long)p.P_max * ((p.L_max + 63) / 64);
    s.splits = (int)std::max<long long>(1, std::min<long long>((512 + wgs - 1) / wgs, tiles / 8));
  }
  return s;
}

bool quant_group_ok(int G) { return G >= 1 && G <= 32; }

size_t quant_attn_scratch(const skip_problem_t& p, int heads_kv) {
  const QuantShape s = quant_shape(p, heads_kv);
  if (s.splits <= 1) return 0;
  return (size_t)p.B * heads_kv * s.chunks * s.splits *
         part_floats(s.rows_chunk * (p.H / heads_kv), p.d_h) * sizeof(float);
}

hipError_t launch_attention_quant(const skip_problem_t& p, const skip_kv_store_t& st,
                                  QuerySource q, const int32_t* kept_offsets,
                                  const int32_t* passage_offsets, const int32_t* passage_blocks,
                                  const int32_t* query_passages, const uint64_t* rowmask,
                                  void* O, float* lse, void* scratch, hipStream_t s) {
  const QuantShape sh = quant_shape(p, st.heads_kv);
  QuantAttnArgs a;
  a.q = static_cast<const bf16_t*>(q.base);
  a.kept_idx = q.kept_idx;
  a.kept_offsets = kept_offsets;
  a.query_passages = query_passages;
  a.passage_offsets = passage_offsets;
  a.passage_blocks = passage_blocks;
  a.rowmask = rowmask;
  a.store = static_cast<const uint8_t*>(st.data);
  a.O = O;
  a.lse = lse;
  a.part = static_cast<float*>(scratch);
  a.n_blocks = st.n_blocks;
  a.N = q.N;
  a.H = p.H;
  a.heads_kv = st.heads_kv;
  a.G = p.H / st.heads_kv;
  a.groups = p.B * st.heads_kv;
  a.chunks = sh.chunks;
  a.splits = sh.splits;
  a.rows_chunk = sh.rows_chunk;
  a.total_kept = p.total_kept;
  a.total_passages = p.total_passages;
  a.total_tokens = p.total_tokens;
  a.k_max = p.k_max;
  a.P_max = p.P_max;
  a.o_f32 = p.o_f32;
  a.scale_log2 = p.sm_scale * kQLog2e;
  const long long wgs = 8 * (((long long)a.groups + 7) / 8) * a.chunks * a.splits;
  if (wgs > (1 << 22)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs);
#define SKIP_ATTN_QUANT(DD, RR, PP)                                                        \
  hipLaunchKernelGGL((attn_quant_kernel<DD, RR, PP>), grid, dim3(kQThreads), 0, s, a)
#define SKIP_ATTN_QUANT_ROWS(DD, PP)                                                       \
  do {                                                                                     \
    if (sh.rows == 192) SKIP_ATTN_QUANT(DD, 192, PP);                                      \
    else if (sh.rows == 64) SKIP_ATTN_QUANT(DD, 64, PP);                                   \
    else SKIP_ATTN_QUANT(DD, 32, PP);                                                      \
  } while (0)
  if (p.d_h == 64) {
    if (p.o_f32) SKIP_ATTN_QUANT_ROWS(64, 3);
    else SKIP_ATTN_QUANT_ROWS(64, 2);
  } else {
    if (p.o_f32) SKIP_ATTN_QUANT_ROWS(128, 3);
    else SKIP_ATTN_QUANT_ROWS(128, 2);
  }
#undef SKIP_ATTN_QUANT_ROWS
#undef SKIP_ATTN_QUANT
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const dim3 mgrid((unsigned)(a.groups * a.chunks));
  if (p.d_h == 64) hipLaunchKernelGGL((attn_quant_merge_kernel<64>), mgrid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attn_quant_merge_kernel<128>), mgrid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace skip
