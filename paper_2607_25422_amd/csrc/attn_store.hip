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
// base 2 and float32.
//
// A unit's (O, max, sum) is merged into the item's, float32 in LDS, in the order
// of the list, so that the result does not depend on which wave was faster: a
// wave waits until every unit of earlier passages and segments is merged.  (Units
// are taken in order, so the earliest one that is not merged never waits.)
//
// A tile of 64 tokens x 32 rows x 128 features takes 128 instructions to make held
// values of codes, some 270 for the softmax and its weights' pieces, and 48 matrix
// products beside them.  16 questions of 192 rows of 32 heads over ten passages of 256
// tokens take 113 us, and no unit is full: vector instructions are active for 52 % of
// the SIMDs' cycles, matrix products for 35 %, and a wave waits for 31 % of its own.  7 us
// of an item's start and end go twice, uncovered (an item's LDS fills a CU), 1.3 a tile and
// SIMD (two waves) and 1.5 a unit, for its queries and its merge.
#include <algorithm>

#include "skip_common.h"
#include "skip_internal.h"
#include "skip_store.h"

namespace skip {

constexpr float kQLog2e = 1.4426950408889634f;
constexpr float kQLn2 = 0.6931471805599453f;
constexpr int kQWaves = 8;
constexpr int kQThreads = 64 * kQWaves;
constexpr int kQMaxP = 64;                 // passages of a question
constexpr int kQRows = 192;                // virtual rows of an item

// Value of lane l ^ 32.
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x),
                                                  false, false);
  return __uint_as_float(__lane_id() < 32 ? r[1] : r[0]);
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

// Adds one to an LDS counter for the whole wave.  The wave barriers keep the branch
// on lane 0 to itself: without them the compiler may join it with another one like
// it across a loop's back edge, and the other lanes run ahead.
__device__ __forceinline__ void wave_add_one(int* counter) {
  __builtin_amdgcn_wave_barrier();
  if (__lane_id() == 0) atomicAdd(counter, 1);
  __builtin_amdgcn_wave_barrier();
}

struct QuantAttnArgs {
  const bf16_t* q;                  // kept rows, or V where kept_idx is given
  const int32_t* kept_idx;
  const int32_t* kept_offsets;
  const int32_t* query_passages;
  const int32_t* passage_offsets;
  const int32_t* passage_blocks;
  const uint64_t* rowmask;          // neighbours of each kept row, or
  const int32_t* edge_rowptr;       // a given graph
  const int32_t* edge_col;
  const uint8_t* store;
  void* O;
  float* lse;
  float* part;                      // partials of split items
  long long n_blocks;
  int B, N, H, heads_kv, G, groups, chunks, splits, rows_chunk;   // rows_chunk: kept rows an item
  int ranked;                       // question_of_rank
  int total_kept, total_passages, total_tokens, total_edges, k_max, P_max, o_f32;
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
// Batches of at most 64 questions whose items differ start with the questions of
// the longest items (rows x tokens of an item; ties: lower index), so that the last
// round of workgroups is a short one: lane b ranks question b.  24 questions of
// mixed sizes, 616 items on 256 CUs: the call 172 us in order, 167 by rank.
__device__ __forceinline__ int question_of_rank(const QuantAttnArgs& a, int r) {
  const int b = min((int)__lane_id(), a.B - 1);
  int k0, k1, p0, p1;
  range_of(a.kept_offsets, b, a.total_kept, k0, k1);
  range_of(a.query_passages, b, a.total_passages, p0, p1);
  const int kq = min(k1 - k0, a.k_max), nch = (kq + a.rows_chunk - 1) / a.rows_chunk;
  const int rpc = nch > 0 ? (kq + nch - 1) / nch : 0;
  const int tok = clampi(a.passage_offsets[p1], 0, a.total_tokens) -
                  clampi(a.passage_offsets[p0], 0, a.total_tokens);
  const float cost = (float)rpc * (float)tok;     // (an order only)
  int rank = 0;
  for (int c = 0; c < a.B; ++c) {
    const float other = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(cost), c));
    rank += (other > cost || (other == cost && c < b)) ? 1 : 0;
  }
  const uint64_t at = __ballot(rank == r && (int)__lane_id() < a.B);
  return __builtin_amdgcn_readfirstlane(at ? __builtin_ctzll(at) : 0);
}
// Chunks and splits of a (question, key head) follow one another on one XCD
// (workgroup id L goes to XCD L % 8), whose L2 then holds its passages once.
template <bool RANKED = false>
__device__ __forceinline__ bool quant_item(const QuantAttnArgs& a, int L, QuantItem& x) {
  const int per = a.chunks * a.splits;
  const int grp = (L & 7) + 8 * ((L >> 3) / per);
  if (grp >= a.groups) return false;
  const int sub = (L >> 3) % per;
  x.chunk = sub / a.splits;
  x.split = sub % a.splits;
  x.b = grp / a.heads_kv;
  x.hk = grp % a.heads_kv;
  if (RANKED && a.ranked) x.b = question_of_rank(a, x.b);
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

// Passages adjacent to a kept row, a bit each (of a given graph here, which saves
// the launch that would write them: 2 us of 10 for one row).  In two steps, so that the
// loads of the first are in flight with the caller's others.
struct RowEdges {
  uint64_t m;
  int e0, e1;
  __device__ __forceinline__ void load(const QuantAttnArgs& a, int row) {
    m = 0ull;
    e0 = e1 = 0;
    if (a.edge_rowptr) {
      e0 = a.edge_rowptr[row];
      e1 = a.edge_rowptr[row + 1];
    } else {
      m = a.rowmask[row];
    }
  }
  __device__ __forceinline__ uint64_t passages(const QuantAttnArgs& a, int P) {
    const uint64_t all = P < 64 ? (1ull << P) - 1ull : ~0ull;
    if (!a.edge_rowptr) return m & all;
    const int b = clampi(e0, 0, a.total_edges), c = clampi(e1, b, a.total_edges);
    constexpr int U = 8;                     // columns in flight
    for (int e = b; e < c; e += U) {
      int j[U];
#pragma unroll
      for (int u = 0; u < U; ++u) j[u] = a.edge_col[min(e + u, c - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j[u] >= 0 && j[u] < P) m |= 1ull << j[u];
    }
    return m;
  }
};
// The question's passage of this lane (lane j: passage j), likewise.
struct LanePassage {
  int t0, t1, blk;
  __device__ __forceinline__ void load(const QuantAttnArgs& a, const QuantItem& it) {
    t0 = t1 = blk = 0;
    const int j = (int)__lane_id();
    if (j < it.P) {
      t0 = a.passage_offsets[it.p0 + j];
      t1 = a.passage_offsets[it.p0 + j + 1];
      blk = a.passage_blocks[it.p0 + j];
    }
  }
  __device__ __forceinline__ int tokens(const QuantAttnArgs& a) const {
    const int b = clampi(t0, 0, a.total_tokens);
    return clampi(t1, b, a.total_tokens) - b;
  }
};

// A tile of 64 tokens: two records of a passage, as a lane holds them.
template <int D>
struct QuantTile {
  static constexpr int C = D / 32, KH = D / 64;   // feature chunks of a record; pairs of them
  static constexpr int FB = D / 32;               // 32-feature blocks of O
  u32x4 k[2][KH], v[FB];
  uint32_t ks, vs;                                // scales, a byte each
  // lane l: n = l % 32, hh = l / 32.  Keys: row n of the two products is token 32
  // kb + 16 h + ki, in features 64 kh + 32 hh ..; values: feature 32 fb + n, tokens
  // 32 hh ..
  // A lane's offsets in a tile whose second record is `step` bytes behind its first
  // (0: the same, masked): of its key row and its values, and of their scales.
  struct Offsets {
    uint32_t k, ks, v, vs;
  };
  static __device__ __forceinline__ Offsets offsets(int n, int hh, uint32_t step) {
    const int ki = 4 * (n >> 3) + (n & 3);        // the lane's key row, of record kb
    const uint32_t kr = ((n >> 2) & 1) ? step : 0u, vr = hh ? step : 0u;
    return {kr + (hh * 16 + ki) * 16, kr + 32 * D + (hh * 16 + ki) * C, vr + n * 16,
            vr + 33 * D + n * C};
  }
  static __device__ __forceinline__ uint32_t scales(const uint8_t* r, uint32_t off) {
    return C == 4 ? *reinterpret_cast<const uint32_t*>(r + off)
                  : *reinterpret_cast<const uint16_t*>(r + off);
  }
  __device__ __forceinline__ void load_k(const uint8_t* r, const Offsets& o) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int kh = 0; kh < KH; ++kh)
        k[h][kh] = *reinterpret_cast<const u32x4*>(r + o.k + (h * C + 2 * kh) * 256);
    ks = scales(r, o.ks);
  }
  __device__ __forceinline__ void load_v(const uint8_t* r, const Offsets& o) {
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
      v[fb] = *reinterpret_cast<const u32x4*>(r + o.v + 16 * D + 512 * fb);
    vs = scales(r, o.vs);
  }
  // S^T: element i of s[h] is token 32 hh + 16 h + i, column n
  __device__ __forceinline__ void logits(const u32x4 (&q)[4 * KH], f32x16_t (&s)[2]) const {
    unrolled<2>([&](auto h_) {
      constexpr int h = decltype(h_)::value;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[h][i] = 0.f;
      unrolled<KH>([&](auto kh_) {
        constexpr int kh = decltype(kh_)::value;
        const float scl = scale_of<h * KH + kh>(ks);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          s[h] = mfma32_bf16(expand8(k[h][kh][c], scl), q[4 * kh + c], s[h]);
      });
    });
  }
  // Weights 2^(sc s - ref), O^T += V^T . P^T; returns the lane's sum of them.  A
  // weight enters as a sum of PIECES bf16 values, all but the last truncated (the
  // rest is exact).
  template <int PIECES>
  __device__ __forceinline__ float weigh(const f32x16_t (&s)[2], float sc, float ref,
                                            f32x16_t (&acc)[FB]) const {
    float ls = 0.f;
    unrolled<4>([&](auto q_) {
      constexpr int q = decltype(q_)::value, h = q >> 1, i0 = 8 * (q & 1);
      u32x4 pc[PIECES];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float p0 = __builtin_amdgcn_exp2f(fmaf(s[h][i0 + 2 * e], sc, -ref));
        float p1 = __builtin_amdgcn_exp2f(fmaf(s[h][i0 + 2 * e + 1], sc, -ref));
        ls += p0 + p1;
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
        const u32x4 va = expand8(v[fb][q], scale_of<fb>(vs));
#pragma unroll
        for (int c = 0; c < PIECES; ++c) acc[fb] = mfma32_bf16(va, pc[c], acc[fb]);
      });
      // (the pieces of one product at a time in registers)
      __builtin_amdgcn_sched_barrier(0);
    });
    return ls;
  }
};

// bf16 pieces of a softmax weight in the second product: two for bf16 output (2^-16
// relative, as in the attention over bf16 passages), three for float output (2^-24).
// One half float a weight (2^-11) would spare bf16 output a third of the products and a
// seventh of the vector instructions (the case above 99 us, 115 with two pieces), but
// not an average that cancels: its own rounding is then far below a weight's.
//
// Weights are 2^(logit - reference), in units of log2; the reference is the largest
// logit so far, kept until one exceeds it by 8.  A unit's reference may lag by that much,
// and the row's that it is merged into by as much again: a weight is at most 2^16 of the
// row's, and 2^31 of them with values below 2^67 sum to less than 2^114.  In a tile with
// larger values the reference is 47 over the largest logit (weights of 2^-31 of the
// row's at most, values below 2^127.6), so that those sums stay finite, too; it is not
// so otherwise, since an exponent of that size is rounded in float32.
template <bool OUT_F32> constexpr int kQPieces = OUT_F32 ? 3 : 2;
constexpr float kQSlack = 8.f;
// Distance from the largest logit to the reference of a tile with these value scales
// (of the lane): 47 where some are 2^65 or more (bytes from 192 on).
__device__ __forceinline__ float over_largest(uint32_t vs) {
  return __any((vs & (vs << 1) & 0x80808080u) != 0u) ? 47.f : 0.f;
}

// Logits of the tokens from `rem` on (of the lane's 32) as -inf.
// (The asm holds the values in their branch: as selects in every tile the compiler
// made them an eighth of the vector instructions.)
__device__ __forceinline__ void mask_from(f32x16_t (&s)[2], int rem) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = 16 * h + i >= rem ? -INFINITY : s[h][i];
      asm volatile("" : "+v"(x));
      s[h][i] = x;
    }
}
__device__ __forceinline__ float lane_max(const f32x16_t (&s)[2]) {
  float lm = s[0][0];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 16; ++i) lm = fmaxf(lm, s[h][i]);
  return lm;
}

// The reference for the next weights (rarely moved: most tiles need no exchange or
// rescale).  lm: the lane's largest logit; over: over_largest of the tile; `first`:
// nothing is summed yet.
template <int FB>
__device__ __forceinline__ void move_ref(float lm, float sc, float over, bool first,
                                         float& m_run, float& l_run, f32x16_t (&acc)[FB]) {
  const float slack = kQSlack - over;
  if (!__any(lm * sc > m_run + slack)) return;
  const float mx = fmaxf(lm, other_half(lm)) * sc;
  const bool up = mx > m_run + slack;
  const float to = mx + over;
  if (!first) {
    const float alpha = !up ? 1.f : m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - to);
    l_run *= alpha;
#pragma unroll
    for (int fb = 0; fb < FB; ++fb) acc[fb] *= alpha;
  }
  m_run = up ? to : m_run;
}

// The reference for weights: where no logit was above -inf so far (products past
// float32), one that leaves them 0 and keeps NaN.
__device__ __forceinline__ float finite_ref(float m_run) { return m_run == -INFINITY ? 0.f : m_run; }

// A stored passage of one key head: its first record, the bytes to the next, its last
// record.  One that is not wholly inside the store is read at record 0 alone.
struct QuantRun {
  const uint8_t* first;
  uint32_t step;
  int last;
  template <int D>
  __device__ __forceinline__ void set(const QuantAttnArgs& a, int hk, int blk, int len) {
    last = max(len - 1, 0) >> 5;
    const bool inside = blk >= 0 && (long long)blk + last < a.n_blocks;
    const uint32_t stride = (uint32_t)a.heads_kv * kStoreRecord<D>;
    step = inside ? stride : 0u;
    first = a.store + (size_t)hk * kStoreRecord<D> + (size_t)(uint32_t)(inside ? blk : 0) * stride;
  }
  // the record of token t (a multiple of 64), and how far behind it the next one
  __device__ __forceinline__ const uint8_t* tile(int t, uint32_t& next) const {
    const int i = min(t >> 5, last);
    next = i < last ? step : 0u;
    return first + (size_t)(uint32_t)i * step;
  }
};

// Result of a virtual row (four features): O, and the LSE with the first.
template <int D>
__device__ __forceinline__ void quant_store(const QuantAttnArgs& a, const QuantItem& it, int i,
                                            int head, int q, float4 o, float m, float l) {
  const float inv = (l == 0.f) ? 0.f : 1.f / l;            // (keeps NaN)
  const size_t at = (size_t)(it.k0 + it.i0 + i) * a.H + head;
  if (a.o_f32)
    *reinterpret_cast<float4*>(static_cast<float*>(a.O) + at * D + q * 4) =
        make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.O) + at * D + q * 4) =
        make_uint2(pack2_bf16(o.x * inv, o.y * inv), pack2_bf16(o.z * inv, o.w * inv));
  if (a.lse && q == 0) a.lse[at] = (l == 0.f) ? -INFINITY : (m + log2f(l)) * kQLn2;
}

template <int D, bool OUT_F32>
__global__ void __launch_bounds__(kQThreads, 2)
attn_quant_kernel(QuantAttnArgs a) {
  constexpr int KH = QuantTile<D>::KH, FB = QuantTile<D>::FB;
  constexpr int NC4 = D / 4;                // 4-float chunks of an accumulator row
  constexpr int ROWS = kQRows, MW = (ROWS + 63) / 64;      // words of a row mask
  constexpr int OS = D + 4;                 // floats of an accumulator row (bank spread)
  __shared__ __attribute__((aligned(16))) float Oacc[ROWS * OS];
  __shared__ float m_acc[ROWS], l_acc[ROWS];
  __shared__ uint64_t neighbours[ROWS];     // of the item's kept rows
  __shared__ uint8_t rowlist[kQMaxP][ROWS]; // virtual rows adjacent to each passage, ascending
  __shared__ int p_cnt[kQMaxP];
  __shared__ int merged;                    // units merged so far

  QuantItem it;
  if (!quant_item<true>(a, blockIdx.x, it)) return;
  const int G = a.G, nv = it.nk * G, P = it.P;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const uint32_t recip_G = (65536u + (uint32_t)G - 1) / (uint32_t)G;   // v / G for v < 192, G <= 32
  auto over_G = [&](int v) -> int { return (int)(((uint32_t)v * recip_G) >> 16); };

  RowEdges edges;
  if (tid < it.nk) edges.load(a, it.k0 + it.i0 + tid);
  LanePassage passage;                      // (every wave the same)
  passage.load(a, it);
  for (int i = tid; i < nv * (OS / 4); i += kQThreads)
    reinterpret_cast<float4*>(Oacc)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = tid; i < nv; i += kQThreads) {
    m_acc[i] = -INFINITY;
    l_acc[i] = 0.f;
  }
  if (tid == 0) merged = 0;
  if (tid < it.nk) neighbours[tid] = edges.passages(a, P);
  const int my_len = passage.tokens(a), my_blk = passage.blk;
  __syncthreads();
  // adjacent rows of each passage, every wave its share of the passages
  uint64_t mk[MW];
#pragma unroll
  for (int w = 0; w < MW; ++w) {
    const int v = 64 * w + lane;
    mk[w] = v < nv ? neighbours[over_G(v)] : 0ull;
  }
  const uint64_t below = (1ull << lane) - 1ull;
  for (int j = wave; j < P; j += kQWaves) {
    int cnt = 0;
#pragma unroll
    for (int w = 0; w < MW; ++w) {
      const bool on = (mk[w] >> j) & 1ull;
      const uint64_t bal = __ballot(on);
      if (on) rowlist[j][cnt + __popcll(bal & below)] = (uint8_t)(64 * w + lane);
      cnt += __popcll(bal);
    }
    if (lane == 0) p_cnt[j] = cnt;
  }

  // The list of units: 32-row blocks of every adjacent passage, each over `segs`
  // equal runs of its tiles (more than one where whole passages would leave waves
  // without a unit).  Every wave forms it (prefix sums of three-bit counts by
  // ballots); wave w takes every eighth unit.
  __syncthreads();
  const int my_cnt = lane < P ? p_cnt[lane] : 0;
  const int my_nblk = my_len > 0 ? (my_cnt + 31) / 32 : 0;
  static_assert(ROWS <= 7 * 32, "blocks of a passage in three bits");
  int blocks = 0, my_first = 0;
#pragma unroll
  for (int bit = 0; bit < 3; ++bit) {
    const uint64_t bal = __ballot((my_nblk >> bit) & 1);
    blocks += __popcll(bal) << bit;
    my_first += __popcll(bal & below) << bit;
  }
  const int segs = blocks >= 2 * kQWaves || blocks == 0
      ? 1 : min((2 * kQWaves + blocks - 1) / blocks, 8);
  my_first *= segs;
  const int u_end = blocks * segs;

  // a sign of the scale, and a scale of 0, are folded into the queries (masked logits
  // stay -inf)
  const uint32_t neg = (a.scale_log2 < 0.f) ? 0x80008000u : 0u;
  const bool flat = a.scale_log2 == 0.f;
  const float sc = flat ? 1.f : fabsf(a.scale_log2);

  struct Unit {
    QuantRun run;
    int t0, t1;                     // tokens
    int before;                     // units to be merged before this one
    int row;                        // this lane's row (-1: none, not merged)
    int src;                        // the kept row, or its visual token
  };
  auto unit = [&](int u, Unit& x) {
    // passage of the unit: the last that starts at or before it (passages
    // without units start where the next one does)
    const int j = __popcll(__ballot(my_first <= u)) - 1;
    const int cnt = __builtin_amdgcn_readlane(my_cnt, j);
    const int len = __builtin_amdgcn_readlane(my_len, j);
    const int uf = __builtin_amdgcn_readlane(my_first, j);
    x.run.template set<D>(a, it.hk, __builtin_amdgcn_readlane(my_blk, j), len);
    const int nblk = (cnt + 31) / 32;
    const int seg = segs == 1 ? 0 : (u - uf) / nblk, m = 32 * ((u - uf) - seg * nblk) + n;
    const int run = ((len + 63) / 64 + segs - 1) / segs * 64;    // tokens of a segment
    x.t0 = min(seg * run, len);
    x.t1 = min(x.t0 + run, len);
    x.before = uf + seg * nblk;
    x.row = m < cnt && x.t0 < x.t1 ? rowlist[j][m] : -1;         // (no tokens: nothing to merge)
    x.src = it.k0 + it.i0 + over_G(max(x.row, 0));
    if (a.kept_idx) x.src = a.kept_idx[x.src];
  };
  u32x4 qf[4 * KH];                          // features 64 kh + 32 hh .. + 31
  auto load_q = [&](const Unit& x) {
    const int v = max(x.row, 0);
    const size_t r = a.kept_idx ? (size_t)it.b * a.N + clampi(x.src, 0, a.N - 1) : (size_t)x.src;
    const bf16_t* src = a.q + (r * a.H + (size_t)(it.hk * G + (v - over_G(v) * G))) * D + 32 * hh;
#pragma unroll
    for (int kh = 0; kh < KH; ++kh)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        qf[4 * kh + s] = *reinterpret_cast<const u32x4*>(src + 64 * kh + 8 * s);
  };
  auto sign_q = [&]() {
    if (neg || flat)
#pragma unroll
      for (int i = 0; i < 4 * KH; ++i) {
        qf[i] = flat ? u32x4{0u, 0u, 0u, 0u} : qf[i] ^ neg;
        asm volatile("" : "+v"(qf[i]));      // (a branch)
      }
  };
  QuantTile<D> x;

  int u = wave;
  Unit cur, nxt;
  if (u < u_end) {
    // (in this order, as in the loop: the counted waits there go by it)
    unit(u, cur);
    load_q(cur);
    asm volatile("" ::: "memory");
    uint32_t next;
    const uint8_t* r = cur.run.tile(cur.t0, next);
    const auto o = x.offsets(n, hh, next);
    x.load_k(r, o);
    asm volatile("" ::: "memory");
    x.load_v(r, o);
    asm volatile("" ::: "memory");
  }
  for (; u < u_end; u += kQWaves) {
    // the next unit's first tile is loaded during this one's last, its queries
    // during the merge
    nxt = cur;
    if (u + kQWaves < u_end) unit(u + kQWaves, nxt);
    // (the queries are waited for here, not in the loop, where the wait would
    // reach the tile's loads, too)
#pragma unroll
    for (int i = 0; i < 4 * KH; ++i) asm volatile("" : "+v"(qf[i]));
    sign_q();
    f32x16_t acc[FB];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[fb][i] = 0.f;
    int t = cur.t0;
    // one tile; the next one's keys (`r`) land during the softmax and the second
    // product, its values during the next logits, and with a unit's last tile the
    // next unit's queries
    auto step = [&](auto last, const uint8_t* r, uint32_t next) {
      f32x16_t s[2];
      x.logits(qf, s);
      const auto o = x.offsets(n, hh, next);
      x.load_k(r, o);
      if constexpr (decltype(last)::value) {
        asm volatile("" ::: "memory");
        load_q(nxt);
        asm volatile("" ::: "memory");
      }
      if (t + 64 > cur.t1) mask_from(s, cur.t1 - t - 32 * hh);
      move_ref(lane_max(s), sc, over_largest(x.vs), t == cur.t0, m_run, l_run, acc);
      l_run += x.template weigh<kQPieces<OUT_F32>>(s, sc, finite_ref(m_run), acc);
      asm volatile("" ::: "memory");
      x.load_v(r, o);
      t += 64;
    };
    uint32_t next;
    while (t + 64 < cur.t1) {
      const uint8_t* r = cur.run.tile(t + 64, next);
      step(std::false_type{}, r, next);
    }
    {                                        // (for an empty segment, too: masked)
      const uint8_t* r = nxt.run.tile(nxt.t0, next);
      step(std::true_type{}, r, next);
    }

    // merge in the order of the list: every unit of earlier passages and
    // segments first (the others of this one have other rows)
    while (__hip_atomic_load(&merged, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) < cur.before)
      __builtin_amdgcn_s_sleep(1);
    asm volatile("" ::: "memory");
    const float l_tot = l_run + other_half(l_run);
    const int row = cur.row;
    if (row >= 0) {
      // (the row's reference moves as a unit's does, so that most merges add only)
      const float mo = m_acc[row], lo = l_acc[row];
      const bool up = m_run > mo + kQSlack;
      const float mn = up ? m_run : mo;
      const float fa = up && mo != -INFINITY ? __builtin_amdgcn_exp2f(mo - mn) : 1.f;
      const float fc = __builtin_amdgcn_exp2f(m_run - finite_ref(mn));   // (0 times 0, or NaN)
      float4* orow = reinterpret_cast<float4*>(Oacc + row * OS) + hh;
      if (__any(fa != 1.f))
#pragma unroll
        for (int c = 0; c < NC4 / 2; ++c) {
          const float4 o = orow[2 * c];
          orow[2 * c] = make_float4(o.x * fa, o.y * fa, o.z * fa, o.w * fa);
        }
      // (a half of the row at a time in registers)
#pragma unroll
      for (int f0 = 0; f0 < FB; f0 += 2) {
        float4 ov[2][4];                     // features 32 fb + 8 c + 4 hh .. + 3
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int c = 0; c < 4; ++c) ov[f][c] = orow[8 * (f0 + f) + 2 * c];
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float4 o = ov[f][c];
            const f32x16_t& x = acc[f0 + f];
            orow[8 * (f0 + f) + 2 * c] =
                make_float4(fmaf(x[4 * c], fc, o.x), fmaf(x[4 * c + 1], fc, o.y),
                            fmaf(x[4 * c + 2], fc, o.z), fmaf(x[4 * c + 3], fc, o.w));
          }
      }
      if (hh == 0) {
        m_acc[row] = mn;
        l_acc[row] = fmaf(l_tot, fc, lo * fa);
      }
    }
    wait_lgkm0();
    wave_add_one(&merged);
    cur = nxt;
  }
  __syncthreads();

  // O = acc / sum for every row, and the LSE (0 and -inf without neighbours)
  for (int e = tid; e < nv * NC4; e += kQThreads) {
    const int ri = e / NC4, q = e % NC4, i = over_G(ri);
    quant_store<D>(a, it, i, it.hk * G + (ri - i * G), q,
                   reinterpret_cast<const float4*>(Oacc + ri * OS)[q],
                   m_acc[ri], l_acc[ri]);
  }
}

// Row-tile form: up to 32 virtual rows a workgroup.  Its waves take the 64-token
// tiles of the passages adjacent to any of the rows in turn, each with its own
// (O, max, sum) in registers from its first tile to its last, so that the loop
// has no LDS, no barrier and one stream of loads a tile ahead; a logit of a row that
// is not adjacent to the tile's passage is -inf (its weight of 0 meets held values,
// which are finite).  The waves' partials are merged in wave order through LDS at the
// end.  Four waves, so that two workgroups share a CU and one starts while the other
// computes (8 questions of 16 heads, 96 rows over 1280 tokens: 28.0 us with the graph,
// 31.3 with eight).  Over long passages: 4 questions of one row of 32 heads over 8 key
// heads and 27000 tokens each, 118 MB of held passages, 30.5 us and 4.3 for the join of
// the parts (3.9 TB/s; matrix products are active for 25 % of the SIMDs' cycles, most of
// them for rows that an item of four rows does not have).
constexpr int kQTileRows = 32;
constexpr int kQTileWaves = 4;
constexpr int kQTileThreads = 64 * kQTileWaves;

template <int D, bool OUT_F32>
__global__ void __launch_bounds__(kQTileThreads, 2)
attn_quant_tile_kernel(QuantAttnArgs a) {
  constexpr int KH = QuantTile<D>::KH, FB = QuantTile<D>::FB, NC4 = D / 4;
  constexpr int OS = D + 4;                 // floats per row of a wave's partial (bank spread)
  __shared__ __attribute__((aligned(16))) float po[kQTileWaves][kQTileRows][OS];
  __shared__ float pm[kQTileWaves][kQTileRows], pl[kQTileWaves][kQTileRows];
  QuantItem it;
  if (!quant_item(a, blockIdx.x, it)) return;
  const int G = a.G, nv = it.nk * G, P = it.P;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;

  // this lane's row (past the item's rows: its last one, adjacent to nothing)
  const int v = min(n, nv - 1), i = v / G, hq = it.hk * G + (v - i * G);
  RowEdges edges;
  edges.load(a, it.k0 + it.i0 + i);
  LanePassage passage;
  passage.load(a, it);
  u32x4 qf[4 * KH];
  {
    const int kr = it.k0 + it.i0 + i;
    const size_t r = a.kept_idx
        ? (size_t)it.b * a.N + clampi(a.kept_idx[kr], 0, a.N - 1) : (size_t)kr;
    const bf16_t* src = a.q + (r * a.H + hq) * D + 32 * hh;
#pragma unroll
    for (int kh = 0; kh < KH; ++kh)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        qf[4 * kh + s] = *reinterpret_cast<const u32x4*>(src + 64 * kh + 8 * s);
  }
  const uint64_t mk = n < nv ? edges.passages(a, P) : 0ull;
  const int my_len = passage.tokens(a), my_blk = passage.blk;
  uint64_t U = mk;                           // passages adjacent to some row
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) U |= (uint64_t)__shfl_xor((unsigned long long)U, s, kWave);
  // tiles of the adjacent passages, one after the other
  const int my_tiles = lane < P && ((U >> lane) & 1ull) ? (my_len + 63) / 64 : 0;
  int my_end = my_tiles;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const int y = __shfl_up(my_end, s, kWave);
    if (lane >= s) my_end += y;
  }
  const int my_first = my_end - my_tiles;
  const int tiles = __builtin_amdgcn_readlane(my_end, kWave - 1);
  const int x0 = (int)((long long)tiles * it.split / a.splits);
  const int x1 = (int)((long long)tiles * (it.split + 1) / a.splits);

  // a sign of the scale, and a scale of 0, are folded into the queries (masked logits
  // stay -inf)
  const uint32_t neg = (a.scale_log2 < 0.f) ? 0x80008000u : 0u;
  const bool flat = a.scale_log2 == 0.f;
  const float sc = flat ? 1.f : fabsf(a.scale_log2);
  struct Place {
    int j, t, len;
    QuantRun run;
  };
  auto place = [&](int c, Place& w) {
    w.j = __popcll(__ballot(my_first <= c)) - 1;         // as for the units above
    w.len = __builtin_amdgcn_readlane(my_len, w.j);
    w.run.template set<D>(a, it.hk, __builtin_amdgcn_readlane(my_blk, w.j), w.len);
    w.t = (c - __builtin_amdgcn_readlane(my_first, w.j)) * 64;
  };
  auto load = [&](const Place& w, QuantTile<D>& x) {
    uint32_t next;
    const uint8_t* r = w.run.tile(w.t, next);
    const auto o = x.offsets(n, hh, next);
    x.load_k(r, o);
    x.load_v(r, o);
    asm volatile("" ::: "memory");           // (tiles in order: the counted waits go by it)
  };
#pragma unroll
  for (int e = 0; e < 4 * KH; ++e) {
    qf[e] = flat ? u32x4{0u, 0u, 0u, 0u} : qf[e] ^ neg;
    asm volatile("" : "+v"(qf[e]));         // (waited for here, not in the loop)
  }
  // whether some query element is 2^100 or more: with all of them below, products
  // with keys below 8 (scale bytes below 128) stay finite
  uint32_t qm = 0u;
#pragma unroll
  for (int e = 0; e < 4 * KH; ++e)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      qm = max(qm, max((qf[e][c] & 0x7fffu) << 16, qf[e][c] & 0x7fff0000u));
  const bool large = __any(qm >= (227u << 23));
  f32x16_t acc[FB];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int fb = 0; fb < FB; ++fb)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[fb][e] = 0.f;
  QuantTile<D> x;
  // its logits into weights; returns the reference of their exponents
  // (a row that is not adjacent: every weight 2^-inf = 0; its logits are set to
  // -inf only where they may be no numbers or +inf, which spares 32 selects a tile)
  auto attend = [&](const Place& w, uint32_t ks, f32x16_t (&s)[2]) -> float {
    if (w.t + 64 > w.len) mask_from(s, w.len - w.t - 32 * hh);
    const bool adj = (mk >> w.j) & 1ull;
    if (large || __any((ks & 0x80808080u) != 0u)) mask_from(s, adj ? 32 : 0);
    move_ref(adj ? lane_max(s) : -INFINITY, sc, over_largest(x.vs), false, m_run, l_run, acc);
    return adj ? finite_ref(m_run) : INFINITY;
  };
  // one tile in registers; the next one's keys land during the softmax, its values
  // during the next logits
  Place w, nw;
  int c = x0 + wave;
  if (c < x1) {
    place(c, w);
    load(w, x);
  }
  for (; c < x1; c += kQTileWaves) {
    f32x16_t s[2];
    x.logits(qf, s);
    const uint32_t ks = x.ks;
    place(min(c + kQTileWaves, x1 - 1), nw);   // (past the last tile: one that is not used)
    uint32_t next;
    const uint8_t* r = nw.run.tile(nw.t, next);
    const auto o = x.offsets(n, hh, next);
    x.load_k(r, o);
    const float ref = attend(w, ks, s);
    l_run += x.template weigh<kQPieces<OUT_F32>>(s, sc, ref, acc);
    asm volatile("" ::: "memory");
    x.load_v(r, o);
    w = nw;
  }

  const float l_tot = l_run + other_half(l_run);
  if (hh == 0) {
    pm[wave][n] = m_run;
    pl[wave][n] = l_tot;
  }
#pragma unroll
  for (int fb = 0; fb < FB; ++fb)
#pragma unroll
    for (int q = 0; q < 4; ++q)              // features 32 fb + 8 q + 4 hh .. + 3
      *reinterpret_cast<float4*>(&po[wave][n][32 * fb + 8 * q + 4 * hh]) =
          make_float4(acc[fb][4 * q], acc[fb][4 * q + 1], acc[fb][4 * q + 2], acc[fb][4 * q + 3]);
  __syncthreads();
  float* part = a.part + ((size_t)((it.b * a.heads_kv + it.hk) * a.chunks + it.chunk) * a.splits +
                          it.split) * part_floats(a.rows_chunk * G, D);
  for (int e = tid; e < nv * NC4; e += kQTileThreads) {
    const int ri = e / NC4, q = e % NC4;
    float M = pm[0][ri];
#pragma unroll
    for (int w = 1; w < kQTileWaves; ++w) M = fmaxf(M, pm[w][ri]);
    const float ref = finite_ref(M);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kQTileWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(pm[w][ri] - ref);
      const float4 y = *reinterpret_cast<const float4*>(&po[w][ri][4 * q]);
      l = fmaf(pl[w][ri], f, l);
      o = make_float4(fmaf(y.x, f, o.x), fmaf(y.y, f, o.y), fmaf(y.z, f, o.z), fmaf(y.w, f, o.w));
    }
    if (a.splits > 1) {
      reinterpret_cast<float4*>(part)[e] = o;
      if (q == 0) {
        part[(size_t)a.rows_chunk * G * D + ri] = M;
        part[(size_t)a.rows_chunk * G * (D + 1) + ri] = l;
      }
    } else {
      const int ii = ri / G;
      quant_store<D>(a, it, ii, it.hk * G + (ri - ii * G), q, o, M, l);
    }
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
    // (eight parts in flight; the maximum moves from batch to batch)
    constexpr int U = 8;
    float M = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < S; s0 += U) {
      float m[U], ls[U];
      float4 x[U];
#pragma unroll
      for (int c = 0; c < U; ++c) {
        const size_t s = (size_t)min(s0 + c, S - 1) * step;
        m[c] = pm[s + ri];
        ls[c] = pl[s + ri];
        x[c] = reinterpret_cast<const float4*>(po + s)[e];
      }
      float mx = M;
#pragma unroll
      for (int c = 0; c < U; ++c) mx = fmaxf(mx, m[c]);
      // (no part with a tile of this row yet: every factor 0, which keeps NaN)
      const float ref = finite_ref(mx), f0 = __builtin_amdgcn_exp2f(M - ref);
      M = mx;
      l *= f0;
      o = make_float4(o.x * f0, o.y * f0, o.z * f0, o.w * f0);
#pragma unroll
      for (int c = 0; c < U; ++c) {
        const float f = s0 + c < S ? __builtin_amdgcn_exp2f(m[c] - ref) : 0.f;
        l = fmaf(ls[c], f, l);
        o = make_float4(fmaf(x[c].x, f, o.x), fmaf(x[c].y, f, o.y), fmaf(x[c].z, f, o.z),
                        fmaf(x[c].w, f, o.w));
      }
    }
    quant_store<D>(a, it, ri / G, it.hk * G + ri % G, q, o, M, l);
  }
}

// How a problem is cut: virtual rows of an item, chunks of a question, splits of
// an item's list.
struct QuantShape {
  bool tile;
  int rows, chunks, rows_chunk, splits;
};
static QuantShape quant_shape(const skip_problem_t& p, int heads_kv) {
  const int G = p.H / heads_kv;
  const long long groups = (long long)p.B * heads_kv;
  QuantShape s;
  auto cut = [&](int rows) {
    s.rows = rows;
    s.rows_chunk = std::max(1, rows / G);
    s.chunks = (p.k_max + s.rows_chunk - 1) / s.rows_chunk;
    return groups * s.chunks;
  };
  s.splits = 1;
  // Row tiles up to three rounds of workgroups for batches of one size (by the average
  // rows of a question): they compute a product for every row and passage that one of
  // their rows has an edge to, the units only those with an edge, in longer items.  Of
  // 90 batches of 1 to 24 questions of 4 to 384 rows this picked the slower form by
  // 1.4 % on average.  32 heads of 128 features, ten passages of 256 tokens, tiles
  // and units: 2 questions of 192 rows (384 tiles) 32 and 47 us, 4 of 96 (384) 33 and
  // 32, 8 of 48 (512) 37 and 30, 8 of 96 (768) 54 and 40, 8 of 192 (1536) 99 and 57.
  const long long per = ((long long)p.total_kept * G + 32ll * p.B - 1) / (32ll * p.B);
  s.tile = groups * per < 768;
  if (!s.tile) {
    cut(kQRows);
    return s;
  }
  const long long wgs = cut(kQTileRows);
  if (wgs > 0 && wgs < 256) {
    // one workgroup a CU, at least four tiles of 64 tokens each: 8 questions of 4 rows
    // and heads over ten passages of 2048 tokens, 32 items, take 108 us whole, 25 in 8
    // parts, 26 in 16; from one part to two a second launch is paid for by 16 tiles
    const long long tiles = (long long)p.P_max * ((p.L_max + 63) / 64);
    if (tiles >= 16) s.splits = (int)std::max<long long>(1, std::min<long long>(256 / wgs, tiles / 4));
  }
  return s;
}

bool quant_group_ok(int G) { return G >= 1 && G <= 32; }

// Workgroups of the attention's launch (a question's and key head's follow one another on
// one XCD), and whether one grid dimension holds them.
static long long quant_workgroups(const skip_problem_t& p, int heads_kv, const QuantShape& s) {
  return 8 * (((long long)p.B * heads_kv + 7) / 8) * s.chunks * s.splits;
}
bool quant_attn_fits(const skip_problem_t& p, int heads_kv) {
  return quant_workgroups(p, heads_kv, quant_shape(p, heads_kv)) <= (1 << 22);
}

size_t quant_attn_scratch(const skip_problem_t& p, int heads_kv) {
  const QuantShape s = quant_shape(p, heads_kv);
  if (s.splits <= 1) return 0;
  return (size_t)p.B * heads_kv * s.chunks * s.splits *
         part_floats(s.rows_chunk * (p.H / heads_kv), p.d_h) * sizeof(float);
}

hipError_t launch_attention_quant(const skip_problem_t& p, const skip_kv_store_t& st,
                                  QuerySource q, const int32_t* kept_offsets,
                                  const int32_t* passage_offsets, const int32_t* passage_blocks,
                                  const int32_t* query_passages, QuantGraph graph, void* O,
                                  float* lse, void* scratch, hipStream_t s) {
  const QuantShape sh = quant_shape(p, st.heads_kv);
  QuantAttnArgs a;
  a.q = static_cast<const bf16_t*>(q.base);
  a.kept_idx = q.kept_idx;
  a.kept_offsets = kept_offsets;
  a.query_passages = query_passages;
  a.passage_offsets = passage_offsets;
  a.passage_blocks = passage_blocks;
  a.rowmask = graph.rowmask;
  a.edge_rowptr = graph.rowptr;
  a.edge_col = graph.col;
  a.total_edges = p.total_edges;
  a.store = static_cast<const uint8_t*>(st.data);
  a.O = O;
  a.lse = lse;
  a.part = static_cast<float*>(scratch);
  a.n_blocks = st.n_blocks;
  a.B = p.B;
  a.N = q.N;
  a.H = p.H;
  a.heads_kv = st.heads_kv;
  a.G = p.H / st.heads_kv;
  a.groups = p.B * st.heads_kv;
  a.chunks = sh.chunks;
  a.splits = sh.splits;
  a.rows_chunk = sh.rows_chunk;
  // (questions of one size: total_kept and total_tokens are B times the largest)
  a.ranked = !sh.tile && p.B > 1 && p.B <= 64 &&
             ((int64_t)p.total_kept < (int64_t)p.B * p.k_max ||
              (int64_t)p.total_tokens < (int64_t)p.B * p.P_max * p.L_max);
  a.total_kept = p.total_kept;
  a.total_passages = p.total_passages;
  a.total_tokens = p.total_tokens;
  a.k_max = p.k_max;
  a.P_max = p.P_max;
  a.o_f32 = p.o_f32;
  a.scale_log2 = p.sm_scale * kQLog2e;
  const dim3 grid((unsigned)quant_workgroups(p, st.heads_kv, sh));
#define SKIP_ATTN_QUANT(DD, FF)                                                            \
  do {                                                                                     \
    if (sh.tile)                                                                           \
      hipLaunchKernelGGL((attn_quant_tile_kernel<DD, FF>), grid, dim3(kQTileThreads), 0, s, a); \
    else                                                                                   \
      hipLaunchKernelGGL((attn_quant_kernel<DD, FF>), grid, dim3(kQThreads), 0, s, a); \
  } while (0)
  if (p.d_h == 64) {
    if (p.o_f32) SKIP_ATTN_QUANT(64, true);
    else SKIP_ATTN_QUANT(64, false);
  } else {
    if (p.o_f32) SKIP_ATTN_QUANT(128, true);
    else SKIP_ATTN_QUANT(128, false);
  }
#undef SKIP_ATTN_QUANT
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const dim3 mgrid((unsigned)(a.groups * a.chunks));
  if (p.d_h == 64) hipLaunchKernelGGL((attn_quant_merge_kernel<64>), mgrid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attn_quant_merge_kernel<128>), mgrid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace skip
