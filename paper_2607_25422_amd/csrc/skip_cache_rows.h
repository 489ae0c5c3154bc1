// Attention of new tokens over a paged cache.
//
// For the new token at position t of a sequence and query head h, with key head h / G,
//   e_m = sm_scale <q_h, K_m>,  O = softmax(e) . V,  LSE = log sum exp e
// over the sequence's tokens m <= t, or over those of them that lie in the pages
// listed for the token and its key head.
//
// A (row, query head of the group) pair is one virtual row: virtual row v of a set of
// rows is its row v / G and query head v % G, and all of them meet the same keys.  An
// item is up to 16 R virtual rows of one key head and one range of tokens:
//   - the tokens of a sequence behind its shared prefix, for its rows (the prefix, for
//     the rows of all sequences of a run that shares it, is skip_cache_tall.h's work);
//   - the listed pages of one row.
// Its tokens are taken in tiles of 32 (a page holds a multiple of that), and a
// wave computes a tile alone, with no barrier:
//   S^T (32 tokens x 16 R rows) = K . Q^T,  O^T (D x 16 R) += V^T . P^T
// (v_mfma_f32_16x16x32_bf16).  Lane l is n = l % 16, g = l / 16.  Which token a row
// of the first product stands for is free: row r of product a is token
// 8 (r / 4) + 4 a + r % 4, so that lane (n, g) holds the logits of tokens 8 g .. + 7 for
// virtual row n, as the second product takes its weights.  Which feature a row of
// the second product stands for is free as well: row n of product i is feature
// (D / 16) n + i, so that a lane takes the same D / 16 features of eight tokens with
// eight loads, and pairs of tokens are joined by byte permutes.  The softmax is
// online, in base 2 and float32.
//
// Work is split evenly whatever the lengths are: all tiles of all items, in order,
// are cut into equal runs, one a workgroup, whose four waves take every fourth tile.
// An item that a run does not hold whole leaves partial results (O, reference, sum),
// which a second kernel joins in the order of the tokens, so that the result does
// not depend on which workgroup was faster.  (More of the split beside kOwnStart.)
//
// The memory bounds it: a tile's keys and values are read once, for whatever rows
// there are, and its loads are in flight during the tile before it.  48 sequences of 300
// to 16384 tokens, 32 heads of 128 over 8: 160 us for 899 MB, 5.6 TB/s, and 5.6 for the
// join.  32 rows of 32 pages of 64 tokens each, the same heads: 54 us for 268 MB, 5.0
// TB/s, and 4.7.  (Loads of two tiles in flight: 196 us against 169; more runs, 768 to
// 4096: 165 to 179 against 162.)
#pragma once

#include "skip_cache.h"
#include "skip_common.h"

namespace skip {

constexpr float kCLog2e = 1.4426950408889634f;
constexpr int kCWaves = 4;
constexpr int kCThreads = 64 * kCWaves;
constexpr int kCTile = kOwnTile;           // tokens of a tile
constexpr int kCLeast = 8;                 // tiles of a run, at least

// bf16 pieces of a softmax weight in the second product: two for bf16 output (2^-16
// relative, as in the attention over passages), three for float output (2^-24).
template <bool OUT_F32> constexpr int kCPieces = OUT_F32 ? 3 : 2;

struct CacheAttnArgs {
  CacheBatch batch;
  CacheView cache;
  CacheResults res;                 // (where results are joined)
  const bf16_t* q;
  const int32_t* pages;             // listed pages [rows][heads_kv][n_sel], or NULL
  void* O;
  float* lse;
  int n_sel, o_f32, runs, direct;
  float scale_log2;
};

// What a run's part of an item is: tiles t0 .. t1 - 1 of its nt.
struct CacheItem {
  int hk, b;                        // key head; the sequence whose pages are read
  int r0, v0, nv;                   // first row; virtual rows v0 .. v0 + nv - 1
  int lo, hi, nt, t0, t1;
  int n;                            // the sequence's new tokens
  bool shared;                      // rows with a prefix: results are joined
};

// What a workgroup keeps in LDS: a wave's keys in turn (see koff), or its results.
template <int D, int R>
struct RowsShared {
  static constexpr int COLS = 16 * R, OS = D + 4;
  static constexpr int PART = COLS * OS * 4 > kCTile * 2 * D ? COLS * OS * 4 : kCTile * 2 * D;
  uint8_t turn[kCWaves][PART];
  float pm[kCWaves][COLS], pl[kCWaves][COLS];
};

// The work of workgroup `block`.  SOLO: every wave takes an item of its own (its partial
// is the whole).
template <int D, int R, bool OUT_F32, bool LISTED, bool SOLO>
__device__ __forceinline__ void cache_rows(const CacheAttnArgs& a, RowsShared<D, R>& sh,
                                           const int block) {
  const CacheBatch& bt = a.batch;
  constexpr int COLS = 16 * R, KC = D / 32, NB = D / 16, FPL = D / 16, PIECES = kCPieces<OUT_F32>;
  constexpr int VW = FPL / 2;               // dwords of a lane's features of a token
  constexpr int OS = D + 4;
  auto& turn = sh.turn;
  auto& pm = sh.pm;
  auto& pl = sh.pl;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int shift = a.cache.shift, hkv = a.cache.heads_kv;

  // a sign of the scale, and a scale of 0, are folded into the queries
  const uint32_t neg = (a.scale_log2 < 0.f) ? 0x80008000u : 0u;
  const bool flat = a.scale_log2 == 0.f;
  const float sc = flat ? 1.f : fabsf(a.scale_log2);

  // Keys come in rows (lane l: 16 bytes of token l / (D / 8)), so that a load takes whole
  // lines, and change hands through the wave's part of LDS: 16 bytes of 16 tokens each,
  // as a product takes them, are as many accesses of the L1 cache (130 rows of 16 heads
  // of d_h 64 over 17 pages of 32 tokens: 44 us, 27 by rows).  Chunk c of token t lies at
  // c ^ (t % 4 + 4 (t / 8 % 2)): eight lanes of a read are eight such tokens.
  constexpr int CH = D / 8, RI = 64 / CH, NI = kCTile / RI;   // chunks; tokens a load; loads
  const int koff = (lane / CH) * D + 8 * (lane % CH);
  const int voff = 8 * g * D + FPL * n;
  const uint32_t klds = lds_addr(turn[wave]);
  auto key_at = [](int t, int c) -> uint32_t {
    return t * 2 * D + 16 * (c ^ ((t & 3) | ((t >> 1) & 4)));
  };
  uint32_t kread[KC];                        // of product 0 (product 1: four tokens on)
#pragma unroll
  for (int c = 0; c < KC; ++c) kread[c] = klds + key_at(8 * (n >> 2) + (n & 3), 4 * c + g);

  // One part of an item: every wave its tiles, then the waves' results together.
  auto work = [&](const CacheItem& it) {
    // this lane's columns: rows, how many tokens they see
    int lim[R];
    u32x4 qf[R][KC];
    const int nblk = (it.nv + 15) / 16;
    auto live = [&](int r) { return R == 1 || r < nblk; };
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int v = it.v0 + min(16 * r + n, it.nv - 1);
      const int ri = v / bt.G, row = it.r0 + ri;
      const bf16_t* src = a.q + ((size_t)row * bt.H + it.hk * bt.G + (v - ri * bt.G)) * D + 8 * g;
      if (live(r))
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          qf[r][c] = *reinterpret_cast<const u32x4*>(src + 32 * c);
          if (neg || flat) qf[r][c] = flat ? u32x4{0u, 0u, 0u, 0u} : qf[r][c] ^ neg;
        }
      lim[r] = LISTED ? it.hi : min(it.hi, it.hi - it.n + ri + 1);   // (hi: the length)
    }
    int least = lim[0], most = lim[0];
#pragma unroll
    for (int r = 1; r < R; ++r) {
      least = min(least, lim[r]);
      most = max(most, lim[r]);
    }
#pragma unroll
    for (int st = 1; st < 16; st <<= 1) {
      least = min(least, __shfl_xor(least, st, kWave));
      most = max(most, __shfl_xor(most, st, kWave));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);

    f32x4_t acc[R][NB];
    float m_run[R], l_run[R];
    bool any_far[R];                         // a row's reference is far (see kCacheFar)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      any_far[r] = false;
      m_run[r] = -INFINITY;
      l_run[r] = 0.f;
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[r][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    u32x4 kf[NI];
    uint32_t vf[8][VW];
    auto load_k = [&](const bf16_t* kp) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        kf[i] = *reinterpret_cast<const u32x4*>(kp + koff + i * RI * D);
    };
    auto load_v = [&](const bf16_t* vp) {
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        if constexpr (VW == 4) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(vp + voff + t * D);
#pragma unroll
          for (int w = 0; w < VW; ++w) vf[t][w] = x[w];
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(vp + voff + t * D);
          vf[t][0] = x.x;
          vf[t][1] = x.y;
        }
      }
    };

    // 64 of the wave's tiles at a time, one a lane: where the tile lies, and its
    // first token
    constexpr int SIDE = SOLO ? 1 : kCWaves;        // waves side by side
    for (int u0 = it.t0 + (SOLO ? 0 : wave); u0 < it.t1; u0 += 64 * SIDE) {
      const int u = u0 + SIDE * lane;
      int at = -1, tok = 0;
      if (u < it.t1) {
        if constexpr (LISTED) {
          const int per = 1 << (shift - 5), e = u / per;
          const int j = a.pages[((size_t)it.r0 * hkv + it.hk) * a.n_sel + e];
          tok = (j << shift) + (u - e * per) * kCTile;
          if (j >= 0 && j <= (it.hi - 1) >> shift && tok < it.hi) at = a.cache.page(it.b, j);
        } else {
          tok = (it.lo / kCTile + u) * kCTile;
          if (tok < most) at = a.cache.page(it.b, tok >> shift);
        }
      }
      uint64_t todo = __ballot(at >= 0);
      if (!todo) continue;
      auto where = [&](int l, int& t) -> size_t {
        t = __builtin_amdgcn_readlane(tok, l);
        return a.cache.base<D>(__builtin_amdgcn_readlane(at, l), it.hk) +
               (size_t)(t & ((1 << shift) - 1)) * D;
      };
      int t;
      size_t off = where(__builtin_ctzll(todo), t);
      load_k(a.cache.k + off);
      asm volatile("" ::: "memory");
      load_v(a.cache.v + off);
      asm volatile("" ::: "memory");
      while (todo) {
        todo &= todo - 1;
        int t_next = t;
        const size_t next = todo ? where(__builtin_ctzll(todo), t_next) : off;
        // logits
        f32x4_t s[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (live(r))
#pragma unroll
            for (int h = 0; h < 2; ++h) s[r][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NI; ++i)
          *reinterpret_cast<u32x4*>(turn[wave] + key_at(RI * i + lane / CH, lane % CH)) = kf[i];
        asm volatile("" ::: "memory");
        // (in turn: a product does not wait for the one before it)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          u32x4 k[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)          // (four tokens on: the same place in a row)
            k[h] = *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)(
                kread[c] + h * 8 * D);
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (live(r))
#pragma unroll
              for (int h = 0; h < 2; ++h) s[r][h] = mfma16_bf16(k[h], qf[r][c], s[r][h]);
        }
        // (the next tile's keys land during the softmax and the second product, its
        // values during the next logits)
        asm volatile("" ::: "memory");
        load_k(a.cache.k + next);
        asm volatile("" ::: "memory");
        if (t < it.lo || t + kCTile > least) {
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (live(r))
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int m = t + 8 * g + e;
              float x = m >= it.lo && m < lim[r] ? s[r][e >> 2][e & 3] : -INFINITY;
              asm volatile("" : "+v"(x));
              s[r][e >> 2][e & 3] = x;
            }
          // values that no row sees are left out
          bool odd = false;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int m = t + 8 * g + e;
            const bool in = m >= it.lo && m < most;
#pragma unroll
            for (int w = 0; w < VW; ++w) {
              uint32_t x = in ? vf[e][w] : 0u;
              asm volatile("" : "+v"(x));
              vf[e][w] = x;
              odd |= bf16_odd_pair(x) != 0u;
            }
          }
          // of the others, a weight of 0 must not meet an infinity or NaN: these are left
          // out, too, and make NaN of the rows that see them (as one product more finds
          // them, of ones)
          if (__any(odd)) {
#pragma unroll
            for (int i = 0; i < NB; ++i) {
              u32x4 ones;
#pragma unroll
              for (int w = 0; w < 4; ++w)
                ones[w] = bf16_odd_pair(__builtin_amdgcn_perm(
                    vf[2 * w + 1][i / 2], vf[2 * w][i / 2], i & 1 ? 0x07060302u : 0x05040100u)) &
                    0x3f803f80u;
#pragma unroll
              for (int r = 0; r < R; ++r) {
                if (!live(r)) continue;
                u32x4 sees;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                  const int m = t + 8 * g + 2 * w;
                  sees[w] = (m >= it.lo && m < lim[r] ? 0x3f80u : 0u) |
                            (m + 1 >= it.lo && m + 1 < lim[r] ? 0x3f800000u : 0u);
                }
                const f32x4_t found = mfma16_bf16(ones, sees, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[r][i][k] += found[k] > 0.f ? NAN : 0.f;
              }
              __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
              for (int w = 0; w < VW; ++w) vf[e][w] &= ~bf16_odd_pair(vf[e][w]);
          }
        }
        // weights 2^(sc s - reference); the reference is over the largest logit that moved
        // it, so that weights are at most 1
        u32x4 pc[R][PIECES];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (!live(r)) continue;
          float lm = s[r][0][0];
#pragma unroll
          for (int e = 1; e < 8; ++e) lm = fmaxf(lm, s[r][e >> 2][e & 3]);
          if (__any(lm * sc > m_run[r])) {
            const float mx = over_groups(lm, [](float x, float y) { return fmaxf(x, y); }) * sc;
            const bool up = mx > m_run[r];
            const float to = up ? cache_reference(mx) : m_run[r];
            const float alpha = !up ? 1.f : m_run[r] == -INFINITY ? 0.f
                                            : __builtin_amdgcn_exp2f(m_run[r] - to);
            l_run[r] *= alpha;
#pragma unroll
            for (int i = 0; i < NB; ++i) acc[r][i] *= alpha;
            m_run[r] = to;
            any_far[r] = __any(cache_far(to));
          }
          float ref = finite_reference(m_run[r]);
          if (__builtin_expect(any_far[r], 0)) {
            const bool far = cache_far(ref);
            const float back = far_back(sc);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              s[r][e >> 2][e & 3] = far_logit(s[r][e >> 2][e & 3], sc, ref, back, far);
            ref = far ? 0.f : ref;
          }
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            float p0 = __builtin_amdgcn_exp2f(fmaf(s[r][w >> 1][2 * (w & 1)], sc, -ref));
            float p1 = __builtin_amdgcn_exp2f(fmaf(s[r][w >> 1][2 * (w & 1) + 1], sc, -ref));
            l_run[r] += p0 + p1;
#pragma unroll
            for (int c = 0; c + 1 < PIECES; ++c) {
              const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
              pc[r][c][w] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
              p0 -= __uint_as_float(b0 & 0xffff0000u);
              p1 -= __uint_as_float(b1 & 0xffff0000u);
            }
            pc[r][PIECES - 1][w] = pack2_bf16(p0, p1);
          }
        }
        // four features' products in turn
#pragma unroll
        for (int i0 = 0; i0 < NB; i0 += 4) {
          u32x4 va[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w)
              va[i][w] = __builtin_amdgcn_perm(vf[2 * w + 1][(i0 + i) / 2], vf[2 * w][(i0 + i) / 2],
                                               i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (live(r))
#pragma unroll
              for (int c = 0; c < PIECES; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  acc[r][i0 + i] = mfma16_bf16(va[i], pc[r][c], acc[r][i0 + i]);
        }
        asm volatile("" ::: "memory");
        load_v(a.cache.v + next);
        asm volatile("" ::: "memory");
        t = t_next;
        off = next;
      }
    }

    // the waves' results together, and where they go
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!live(r)) continue;
      const float l = over_groups(l_run[r], [](float x, float y) { return x + y; });
      const int col = 16 * r + n;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float* dst = reinterpret_cast<float*>(turn[wave]) + col * OS + FPL * (4 * g + k);
#pragma unroll
        for (int i = 0; i < NB; i += 4)
          *reinterpret_cast<float4*>(dst + i) = make_float4(
              acc[r][i][k], acc[r][i + 1][k], acc[r][i + 2][k], acc[r][i + 3][k]);
      }
      if (g == 0) {
        pm[wave][col] = m_run[r];
        pl[wave][col] = l;
      }
    }
    if (SOLO) wait_lgkm0();
    else __syncthreads();
    constexpr int NC4 = D / 4;
    const bool all = it.t0 == 0 && it.t1 == it.nt;
    const int run = block;
    const int w0 = SOLO ? wave : 0, w1 = SOLO ? wave + 1 : kCWaves;
    for (int e = SOLO ? lane : tid; e < it.nv * NC4; e += SOLO ? 64 : kCThreads) {
      const int col = e / NC4, c4 = e % NC4;
      float m = pm[w0][col];
      if (!SOLO)
#pragma unroll
        for (int w = 1; w < kCWaves; ++w) m = fmaxf(m, pm[w][col]);
      const float ref = m == -INFINITY ? 0.f : m;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
#pragma unroll
      for (int w = w0; w < w1; ++w) {
        const float f = __builtin_amdgcn_exp2f(pm[w][col] - ref);
        const float4 x = *reinterpret_cast<const float4*>(
            reinterpret_cast<const float*>(turn[w]) + col * OS + 4 * c4);
        o.x = fmaf(x.x, f, o.x);
        o.y = fmaf(x.y, f, o.y);
        o.z = fmaf(x.z, f, o.z);
        o.w = fmaf(x.w, f, o.w);
        l = fmaf(pl[w][col], f, l);
      }
      const int v = it.v0 + col, ri = v / bt.G;
      const size_t vr = (size_t)(it.r0 + ri) * bt.H + it.hk * bt.G + (v - ri * bt.G);
      if (all && !it.shared) {
        const float inv = l == 0.f ? 0.f : 1.f / l;            // (keeps NaN)
        if (OUT_F32)
          *reinterpret_cast<float4*>(static_cast<float*>(a.O) + vr * D + 4 * c4) =
              make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        else
          *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.O) + vr * D + 4 * c4) =
              make_uint2(pack2_bf16(o.x * inv, o.y * inv), pack2_bf16(o.z * inv, o.w * inv));
        if (a.lse && c4 == 0) a.lse[vr] = l == 0.f ? -INFINITY : (m + log2f(l)) * kCacheLn2;
      } else {
        float *w, *ml;
        int ml_step;
        if (all) {
          w = whole_at<D>(a.res, bt, 1, vr);
          ml = w + D;
          ml_step = 1;
        } else {
          w = a.res.part + (size_t)(2 * run + (it.t0 == 0 ? 1 : 0)) * part_floats<D>(COLS);
          ml = w + (size_t)COLS * D + col;
          ml_step = COLS;
          w += (size_t)col * D;
        }
        *reinterpret_cast<float4*>(w + 4 * c4) = o;
        if (c4 == 0) {
          ml[0] = m;
          ml[ml_step] = l;
        }
      }
    }
    if (SOLO) wait_lgkm0();
    else if (!a.direct) __syncthreads();       // (the next item's keys take their place)
  };

  if constexpr (LISTED) {
    const int rows = clampi(bt.row_offsets[bt.B], 0, bt.total_rows);
    const int nt = a.n_sel << (shift - 5);
    auto listed = [&](int row, int hk, int t0, int t1) {
      CacheItem it;
      it.r0 = row;
      it.hk = hk;
      it.nt = nt;
      it.t0 = t0;
      it.t1 = t1;
      CacheSeq s;
      it.b = seq_of_row(bt.row_offsets, bt.lens, bt.B, bt.total_rows, bt.k_max, bt.L_max, row, s);
      if (it.b < 0) return;
      it.v0 = 0;
      it.nv = bt.G;
      it.lo = 0;
      it.hi = max(s.len - s.n + row - s.r0 + 1, 0);
      it.n = 1;
      it.shared = false;
      work(it);
    };
    if (a.direct) {
      // An item a workgroup (SOLO: a wave).  Workgroup id L goes to XCD L % 8; rows of
      // one key head stay on one, whose L2 holds the pages that they share (130
      // rows of 16 heads over 17 pages each).
      const int x = block & 7;
      const int i = SOLO ? (block >> 3) * kCWaves + wave : block >> 3;
      int row, hk;
      if (hkv % 8 == 0) {
        row = i / (hkv / 8);
        hk = x + 8 * (i - row * (hkv / 8));
      } else if (8 % hkv == 0) {
        row = i * (8 / hkv) + x / hkv;
        hk = x % hkv;
      } else {
        row = (8 * i + x) / hkv;
        hk = 8 * i + x - row * hkv;
      }
      if (row < rows) listed(row, hk, 0, nt);
      return;
    }
    const int step = nt + kOwnStart, W = rows * hkv * step;
    const int per = max((W + a.runs - 1) / a.runs, kCLeast);
    if (block == 0 && tid == 0) a.res.meta[(size_t)bt.B * kCacheMeta] = per;
    int u = block * per;
    const int end = min(W - u, per) + u;
    while (u < end) {
      const int i = u / step, start = i * step, row = i / hkv;
      const int t0 = tile_at<kOwnStart>(u - start, nt), t1 = tile_at<kOwnStart>(end - start, nt);
      if (t0 < t1) listed(row, i - row * hkv, t0, t1);
      u = start + step;
    }
  } else {
    SeqWalk<false> walk;
    walk.cols = COLS;
    auto own = [&](CacheItem& it, int L) {       // the sequence in lane L
      it.b = walk.sb0 + L;
      it.r0 = walk.of_lane(walk.sb.s.r0, L);
      it.n = walk.of_lane(walk.sb.s.n, L);
      it.hi = walk.of_lane(walk.sb.s.len, L);
      const int P = walk.of_lane(walk.sb.P, L);
      it.lo = min(P, it.hi);
      it.shared = P > 0;
      it.nt = SeqBlock::own_tiles(it.lo, it.hi);
    };
    if (a.direct) {
      // short sequences: an item a workgroup, no parts
      const int rt = (bt.k_max * bt.G + COLS - 1) / COLS;
      const int b = block / (hkv * rt), i = block - b * hkv * rt;
      CacheSeq s;
      s.load(bt.row_offsets, bt.lens, b, bt.total_rows, bt.k_max, bt.L_max);
      CacheItem it;
      it.b = b;
      it.r0 = s.r0;
      it.n = s.n;
      it.hk = i / rt;
      it.v0 = (i - it.hk * rt) * COLS;
      it.nv = min(COLS, s.n * bt.G - it.v0);
      if (it.nv <= 0) return;
      it.lo = 0;
      it.hi = s.len;
      it.nt = SeqBlock::own_tiles(0, s.len);
      it.t0 = 0;
      it.t1 = it.nt;
      it.shared = false;
      work(it);
      return;
    }
    // all tiles, and the places of the items for the join
    int pre_before = 0;
    const int W = walk.total(bt, [&](int before) {
      if (block != 0 || wave != 0) return;
      const SeqBlock& sb = walk.sb;
      const int pre_incl = (int)wave_incl_scan((uint32_t)sb.pre);
      const int pre = __shfl(pre_before + pre_incl - sb.pre, sb.first, kWave);
      const int r_first = __shfl(sb.s.r0, sb.first, kWave);
      if (walk.sb0 + lane < bt.B) {
        int32_t* w = a.res.meta + (size_t)(walk.sb0 + lane) * kCacheMeta;
        reinterpret_cast<int4*>(w)[0] = make_int4(before + walk.incl - sb.own, pre, sb.P, r_first);
        reinterpret_cast<int4*>(w)[1] = make_int4(sb.run_rows, sb.s.r0, sb.s.n, sb.s.len);
      }
      pre_before += __builtin_amdgcn_readlane(pre_incl, 63);
    });
    const int per = max((W + a.runs - 1) / a.runs, kCLeast);
    if (block == 0 && tid == 0) a.res.meta[(size_t)bt.B * kCacheMeta] = per;
    int u = block * per;
    if (u >= W) return;
    const int end = min(W - u, per) + u;
    while (u < end) {
      int first;
      const int L = walk.seek(bt, u, first);
      CacheItem it;
      own(it, L);
      const int step = it.nt + kOwnStart;
      const int rt = SeqBlock::row_tiles(bt, it.n, COLS), i = (u - first) / step;
      it.hk = i / rt;
      it.v0 = (i - it.hk * rt) * COLS;
      it.nv = min(COLS, it.n * bt.G - it.v0);
      const int start = first + i * step;
      it.t0 = tile_at<kOwnStart>(u - start, it.nt);
      it.t1 = tile_at<kOwnStart>(end - start, it.nt);
      u = start + step;
      if (it.t0 < it.t1) work(it);
    }
  }
}

// The launch of shared prefixes' items and sequences' own, results left for the join.
hipError_t launch_cache_shared(const CacheAttnArgs& own, int d_h, int R, hipStream_t s);

}  // namespace skip
