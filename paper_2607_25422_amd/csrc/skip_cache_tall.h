// Attention of new tokens over a paged cache, for sequences with many of them (the
// formulas and the virtual rows are at the top of skip_cache_rows.h).
//
// An item is 128 virtual rows of one sequence (or of the sequences that share a prefix)
// and key head, over the tokens that its last row sees (or the prefix).  A workgroup
// takes one, or an equal run of all items' tiles: its four waves hold 32 virtual rows each
// and share tiles of 64 tokens in LDS, which direct loads fill a tile (d_h 64: two)
// ahead.  Per tile and wave,
//   S^T (64 tokens x 32 rows) = K . Q^T,  O^T (D x 32) += V^T . P^T
// (v_mfma_f32_32x32x16_bf16).  Lane l is n = l % 32, hh = l / 32.  Element i of the
// first product's half h is token 32 h + 8 (i / 4) + 4 hh + i % 4 of row n, and stays
// where it is as a weight: contraction slot (hh, j) of the second product's step
// (h, q) stands for token 32 h + 16 q + 8 (j / 4) + 4 hh + j % 4.  Its V^T operand comes
// out of row-major V by transposing LDS reads (16 lanes take four tokens of 16
// features each way).
//
// A row of LDS is a token's D values in chunks of 16 bytes, at places exchanged by the
// token: chunk c of token r lies at c ^ (r % 16) (keys: eight lanes of a 16-byte read
// are eight tokens) and at c ^ 2 (r % 8) (values: 16 lanes of a transposing read are
// four tokens of 32 bytes).  The direct loads take chunks in that order.
//
// Matrix and vector instructions bound it together: four prompts of 1024 to 4096
// tokens, 32 heads of 128 over 8, take 340 us, 694 TFLOP/s (1040 with the second piece of
// the weights); the matrix units are busy for 49 % of the SIMDs' cycles, vector
// instructions are issued in 45 % of them, two waves a SIMD.  Four prefixes of 8217
// tokens for 16 sequences each, with their own 1 to 500 tokens behind them in one launch:
// 51 us.  Six pieces of 98 to 129 rows over 3102 to 3362 tokens, 16 heads of 64, float output:
// 37 (40 with items sequence by sequence, see the end of the work).
#pragma once

#include "skip_cache.h"
#include "skip_common.h"

namespace skip {

constexpr int kTWaves = 4;
constexpr int kTThreads = 64 * kTWaves;
constexpr int kTRows = 32 * kTWaves;       // virtual rows of an item
constexpr int kTTile = 64;                 // tokens of a tile
constexpr int kTLeast = 4;                 // tiles of a run, at least
// Tokens of a sequence that a workgroup takes whole, rather than in runs with a join
// (480 rows of 481 tokens, 32 heads over 8: 31 us in runs, 17 whole).
constexpr int kTShort = 768;
static_assert(kTRows == kPrefixRows && kTTile == kPrefixTile, "items of prefixes");
template <bool OUT_F32> constexpr int kTPieces = OUT_F32 ? 3 : 2;

struct TallArgs {
  CacheBatch batch;
  CacheView cache;
  CacheResults res;                 // (prefixes)
  const bf16_t* q;
  void* O;
  float* lse;
  int row_tiles, runs, grouped;
  float scale_log2;
};

// What a workgroup works on: 128 virtual rows, tiles i0 .. i1 - 1 of the nt that hold
// the tokens before hi.
struct TallItem {
  int b, hk;                        // the sequence whose pages are read; key head
  int r0, v0, nv;                   // first row of the set; virtual rows v0 .. v0 + nv - 1
  int hi, nt, i0, i1;
  CacheSeq s;
};
// Workgroup id L goes to XCD L % 8; where sequences and key heads make whole eights,
// the items of one of them follow one another on one XCD, whose L2 then holds its keys
// and values.  Row tiles from the last, which see most tokens, to the first.
__device__ __forceinline__ bool tall_item(const TallArgs& a, int L, TallItem& x) {
  const CacheBatch& bt = a.batch;
  const int per = a.row_tiles, groups = bt.B * bt.heads_kv;
  const int grp = a.grouped ? (L & 7) + 8 * ((L >> 3) / per) : L / per;
  const int sub = a.grouped ? (L >> 3) % per : L % per;
  if (grp >= groups) return false;
  x.b = grp / bt.heads_kv;
  x.hk = grp - x.b * bt.heads_kv;
  x.s.load(bt.row_offsets, bt.lens, x.b, bt.total_rows, bt.k_max, bt.L_max);
  const int rts = SeqBlock::row_tiles(bt, x.s.n, kTRows);
  if (sub >= rts) return false;
  const int rt = rts - 1 - sub;
  x.r0 = x.s.r0;
  x.v0 = rt * kTRows;
  x.nv = min(kTRows, x.s.n * bt.G - x.v0);
  // the tokens that the last row sees
  x.hi = max(x.s.len - x.s.n + (x.v0 + x.nv - 1) / bt.G + 1, 0);
  x.nt = (x.hi + kTTile - 1) / kTTile;
  x.i0 = 0;
  x.i1 = x.nt;
  return true;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
// Four values of a column of 4 x 16 ones in LDS (this lane reads a quarter of a row).
__device__ __forceinline__ uint2 lds_read_transposed(uint32_t addr) {
  typedef __attribute__((address_space(3))) s16x4* Ptr;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(uintptr_t)addr));
}
__device__ __forceinline__ u32x4 lds_read16(uint32_t addr) {
  typedef const __attribute__((address_space(3))) u32x4* Ptr;
  return *(Ptr)(uintptr_t)addr;
}

// OF: sequences, an item a workgroup; sequences, in equal runs of tiles; prefixes, in
// equal runs.
enum TallOf { kTallItems, kTallRuns, kTallPrefixes };
// What a workgroup keeps in LDS: tiles, and the bits of clean (below).
template <int D>
struct TallShared {
  static constexpr int ROW = 2 * D, CH = D / 8;     // bytes and chunks of a token
  static constexpr uint32_t kKeys = kTTile * ROW, kBuffer = 2 * kKeys;
  static constexpr uint32_t kBuffers = D == 64 ? 3 : 2;   // (48 KiB: three workgroups a CU; 64: two)
  uint8_t tile[kBuffers * kBuffer];
  uint8_t unseen[kTTile][CH];
  int flags[kTWaves];
};

// The work of workgroup `block` of a launch of a.runs.
template <int D, bool OUT_F32, TallOf OF>
__device__ __forceinline__ void cache_tall_work(const TallArgs& a, TallShared<D>& sh,
                                                const int block) {
  constexpr bool PREFIX = OF == kTallPrefixes;
  const CacheBatch& bt = a.batch;
  constexpr int KC = D / 16, FB = D / 32, PIECES = kTPieces<OUT_F32>;
  typedef TallShared<D> Shared;
  constexpr int ROW = Shared::ROW, CH = Shared::CH;
  constexpr uint32_t kKeys = Shared::kKeys, kBuffer = Shared::kBuffer, kBuffers = Shared::kBuffers;
  auto& tile = sh.tile;
  auto& unseen = sh.unseen;
  auto& flags = sh.flags;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int shift = a.cache.shift;
  const uint32_t lds = lds_addr(tile);
  // (runs that follow one another go to one XCD, whose L2 holds what they share)
  const int run = OF == kTallItems ? 0 : (block & 7) * (a.runs / 8) + (block >> 3);
  SeqWalk<PREFIX, OF == kTallRuns> walk;
  walk.cols = 16;                                   // (own items are not looked at)

  const uint32_t neg = (a.scale_log2 < 0.f) ? 0x80008000u : 0u;
  const bool flat = a.scale_log2 == 0.f;
  const float sc = flat ? 1.f : fabsf(a.scale_log2);
  // LDS addresses of this lane's operands in the first buffer
  uint32_t ka[KC], va_[FB];
#pragma unroll
  for (int c = 0; c < KC; ++c) ka[c] = lds + n * ROW + 16 * ((2 * c + hh) ^ (n & (CH - 1)));
  {
    const int j = lane & 15, fh = (lane >> 4) & 1, r = 4 * hh + (j >> 2);
#pragma unroll
    for (int f = 0; f < FB; ++f) {
      const int c = 4 * f + 2 * fh + ((j & 3) >> 1);
      va_[f] = lds + kKeys + r * ROW + 16 * (c ^ ((2 * r) & (CH - 1))) + 8 * (j & 1);
    }
  }

  // direct loads: the wave takes 16 tokens of each tile, 1 KiB an instruction
  constexpr int RI = 1024 / ROW, NI = 16 / RI;      // tokens an instruction, instructions
  uint32_t kg[NI], vg[NI];                          // source offsets from the 16 tokens (bytes)
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = RI * i + lane / CH, c = lane % CH;          // (r: of 16)
    kg[i] = r * ROW + 16 * (c ^ (r & (CH - 1)));
    vg[i] = r * ROW + 16 * (c ^ ((2 * r) & (CH - 1)));
  }
  auto work = [&](const TallItem& it) {
  // this lane's row and how many tokens it sees; the wave's least and most
  const int wv = it.v0 + 32 * wave;                 // the wave's first virtual row
  const bool any = wv < it.v0 + it.nv;
  const int v = min(wv + n, it.v0 + it.nv - 1);
  const int ri = v / bt.G, head = it.hk * bt.G + (v - ri * bt.G), row = it.r0 + ri;
  int lim, least, most, least_all;
  if constexpr (PREFIX) {
    // the row's sequence: the last of the block that starts at or before it (a sequence
    // without rows starts where the next one does)
    auto limit = [&](int r) -> int {
      int l = 0;
#pragma unroll
      for (int st = 32; st >= 1; st >>= 1)
        if (__shfl(walk.sb.s.r0, l + st, kWave) <= r && walk.sb0 + l + st < bt.B) l += st;
      const int sr0 = __shfl(walk.sb.s.r0, l, kWave), sn = __shfl(walk.sb.s.n, l, kWave);
      const int sl = __shfl(walk.sb.s.len, l, kWave);
      return r < sr0 + sn ? clampi(sl - sn + (r - sr0) + 1, 0, it.hi) : 0;
    };
    lim = limit(row);
    least = most = lim;
    least_all = it.hi;
    for (int u = lane; u - lane < it.nv; u += kWave)
      least_all = min(least_all, limit(it.r0 + (it.v0 + min(u, it.nv - 1)) / bt.G));
#pragma unroll
    for (int st = 1; st < kWave; st <<= 1) {
      least = min(least, __shfl_xor(least, st, kWave));
      most = max(most, __shfl_xor(most, st, kWave));
      least_all = min(least_all, __shfl_xor(least_all, st, kWave));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    least_all = __builtin_amdgcn_readfirstlane(least_all);
  } else {
    const int before = it.s.len - it.s.n + 1;
    lim = max(before + ri, 0);
    least_all = max(before + it.v0 / bt.G, 0);
    least = max(before + min(wv, it.v0 + it.nv - 1) / bt.G, 0);
    most = max(before + min(wv + 31, it.v0 + it.nv - 1) / bt.G, 0);
  }
  u32x4 qf[KC];
  {
    const bf16_t* src = a.q + ((size_t)row * bt.H + head) * D + 8 * hh;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      qf[c] = *reinterpret_cast<const u32x4*>(src + 16 * c);
      if (neg || flat) qf[c] = flat ? u32x4{0u, 0u, 0u, 0u} : qf[c] ^ neg;
    }
  }
  // pages of 64 tiles at a time: lane i those of tile i's two halves
  int pa = 0, pb = 0, pages_from = it.i0;
  auto load_pages = [&]() {
    const int t = (pages_from + lane) * kTTile;
    pa = t < it.hi ? a.cache.page(it.b, t >> shift) : 0;
    pb = t + 32 < it.hi ? a.cache.page(it.b, (t + 32) >> shift) : 0;
  };
  uint32_t missing = 0;                             // halves without a page, by buffer
  // (tokens behind the last one are loaded from where they would lie, and masked)
  auto fetch = [&](int i, uint32_t buffer) {
    if (i - pages_from >= 64) {
      pages_from = i;
      load_pages();
    }
    const int pa_i = __builtin_amdgcn_readlane(pa, i - pages_from);
    const int pb_i = __builtin_amdgcn_readlane(pb, i - pages_from);
    const int own = wave < 2 ? pa_i : pb_i;
    const int at = 2 * (buffer / kBuffer);
    missing = (missing & ~(3u << at)) | (((pa_i < 0 ? 1u : 0u) | (pb_i < 0 ? 2u : 0u)) << at);
    const int t = i * kTTile + 16 * wave;
    const size_t off = a.cache.base<D>(max(own, 0), it.hk) + (size_t)(t & ((1 << shift) - 1)) * D;
    const uint8_t* ks = reinterpret_cast<const uint8_t*>(a.cache.k + off);
    const uint8_t* vs = reinterpret_cast<const uint8_t*>(a.cache.v + off);
    const uint32_t to = lds + buffer + 16 * wave * ROW;
#pragma unroll
    for (int j = 0; j < NI; ++j) lds_dma16(ks + kg[j], to + 1024 * j);
#pragma unroll
    for (int j = 0; j < NI; ++j) lds_dma16(vs + vg[j], to + kKeys + 1024 * j);
  };

  f32x16_t acc[FB];
  float m_run = -INFINITY, l_run = 0.f;
  bool any_far = false;                             // a row's reference is far (see kCacheFar)
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[f][i] = 0.f;

  uint32_t buffer = 0;
  auto compute = [&](bool masked, int t, int miss) {
    f32x16_t s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[h][i] = 0.f;
    // (the two halves' products in turn: neither waits for its own last one)
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        s[h] = mfma32_bf16(lds_read16(ka[c] + buffer + 32 * h * ROW), qf[c], s[h]);
    // four pairs of reads ahead of the products
    __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
      if (c < KC - 4) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    if (masked) {
      // (asm holds what is masked in its branch, and what it is compared with out of
      // registers)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int rem = (miss >> h) & 1 ? 0 : lim - t - 32 * h - 4 * hh;
        asm volatile("" : "+v"(rem));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float x = 8 * (i >> 2) + (i & 3) < rem ? s[h][i] : -INFINITY;
          asm volatile("" : "+v"(x));
          s[h][i] = x;
        }
      }
    }
    float lm = s[0][0];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) lm = fmaxf(lm, s[h][i]);
    if (__any(lm * sc > m_run)) {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(lm), __float_as_uint(lm),
                                                      false, false);
      const float mx = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) * sc;
      const bool up = mx > m_run;
      const float to = up ? cache_reference(mx) : m_run;
      const float alpha = !up ? 1.f : m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - to);
      l_run *= alpha;
#pragma unroll
      for (int f = 0; f < FB; ++f) acc[f] *= alpha;
      m_run = to;
      any_far = __any(cache_far(to));
    }
    float ref = finite_reference(m_run);
    if (__builtin_expect(any_far, 0)) {
      const bool far = cache_far(ref);
      const float back = far_back(sc);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[h][i] = far_logit(s[h][i], sc, ref, back, far);
      ref = far ? 0.f : ref;
    }
    // weights of step (h, q) as bf16 pieces, and its values
    auto weigh = [&](auto step, u32x4 (&pc)[PIECES]) {
      constexpr int h = decltype(step)::value >> 1, q = decltype(step)::value & 1;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float p0 = __builtin_amdgcn_exp2f(fmaf(s[h][8 * q + 2 * w], sc, -ref));
        float p1 = __builtin_amdgcn_exp2f(fmaf(s[h][8 * q + 2 * w + 1], sc, -ref));
        l_run += p0 + p1;
#pragma unroll
        for (int c = 0; c + 1 < PIECES; ++c) {
          const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
          pc[c][w] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
          p0 -= __uint_as_float(b0 & 0xffff0000u);
          p1 -= __uint_as_float(b1 & 0xffff0000u);
        }
        pc[PIECES - 1][w] = pack2_bf16(p0, p1);
      }
    };
    auto values = [&](auto step, u32x4 (&x)[FB]) {
      constexpr int h = decltype(step)::value >> 1, q = decltype(step)::value & 1;
#pragma unroll
      for (int f = 0; f < FB; ++f) {
        const uint32_t at = va_[f] + buffer + (32 * h + 16 * q) * ROW;
        const uint2 lo = lds_read_transposed(at), up = lds_read_transposed(at + 8 * ROW);
        x[f] = u32x4{lo.x, lo.y, up.x, up.y};
      }
    };
    auto product = [&](const u32x4 (&pc)[PIECES], const u32x4 (&x)[FB]) {
#pragma unroll
      for (int c = 0; c < PIECES; ++c)
#pragma unroll
        for (int f = 0; f < FB; ++f) acc[f] = mfma32_bf16(x[f], pc[c], acc[f]);
    };
    // a step's products in turn with the next one's weights, which they hide
    u32x4 pc[2][PIECES], x[2][FB];
    weigh(std::integral_constant<int, 0>{}, pc[0]);
    values(std::integral_constant<int, 0>{}, x[0]);
    unrolled<4>([&](auto step) {
      constexpr int k = decltype(step)::value;
      if constexpr (k < 3) {
        values(std::integral_constant<int, k + 1>{}, x[(k + 1) & 1]);
        weigh(std::integral_constant<int, k + 1>{}, pc[(k + 1) & 1]);
      }
      product(pc[k & 1], x[k & 1]);
    });
  };

  // Values in a tile that some rows do not see: a weight of 0 must not meet an infinity
  // or NaN.  Every wave looks through the 16 tokens that it loaded: what no row sees is
  // zeroed; of the others, what is not finite is zeroed and remembered, a bit a value.
  auto clean = [&](int t, int miss) {
    bool found = false;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int r = 16 * wave + RI * j + lane / CH, c = lane % CH;     // token, place
      const uint32_t at = buffer + kKeys + r * ROW + 16 * c;
      u32x4 x = *reinterpret_cast<const u32x4*>(tile + at);
      const bool seen = t + r < it.hi && !((miss >> (r >> 5)) & 1);
      uint32_t bits = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t bad = seen ? bf16_odd_pair(x[w]) : 0u;
        x[w] &= seen ? ~bad : 0u;
        bits |= (bad & 1u) << (2 * w) | (bad >> 31) << (2 * w + 1);
      }
      *reinterpret_cast<u32x4*>(tile + at) = x;
      unseen[r][c ^ ((2 * r) & (CH - 1))] = (uint8_t)bits;
      found |= bits != 0u;
    }
    const bool any_found = __any(found);
    if (lane == 0) flags[wave] = any_found;
  };
  // NaN to the rows that see such a value, in its feature.
  auto poison = [&](int t) {
#pragma clang loop unroll(disable)
    for (int r = 0; r < kTTile; ++r)
#pragma unroll
      for (int f = 0; f < FB; ++f) {
        uint32_t bits = reinterpret_cast<const uint32_t*>(unseen[r])[f] >> (4 * hh);
        if (t + r >= lim) bits = 0u;
        if (!__any(bits != 0u)) continue;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((bits >> (8 * (i >> 2) + (i & 3))) & 1u) acc[f][i] = NAN;
      }
  };

  if (it.i0 < it.i1) {
    load_pages();
    if constexpr (OF != kTallItems) barrier_lds();       // (the last item's tiles are read)
#pragma unroll
    for (uint32_t j = 0; j + 1 < kBuffers; ++j)
      if (it.i0 + (int)j < it.i1) fetch(it.i0 + j, j * kBuffer);
  }
  for (int i = it.i0; i < it.i1; ++i) {
    // this tile's loads have landed, and every wave is through with the last one, whose
    // place the next one takes
    constexpr int ahead = kBuffers - 2;
    if (i + ahead < it.i1) wait_vmcnt<ahead * 2 * NI>();
    else wait_vmcnt<0>();
    barrier_lds();
    const int miss = (missing >> (2 * (buffer / kBuffer))) & 3;
    if (i + (int)kBuffers - 1 < it.i1)
      fetch(i + kBuffers - 1, (buffer + (kBuffers - 1) * kBuffer) % (kBuffers * kBuffer));
    const int t = i * kTTile;
    bool odd = false;
    if (t + kTTile > least_all || miss) {
      clean(t, miss);
      barrier_lds();
      odd = flags[0] | flags[1] | flags[2] | flags[3];
    }
    if (any && t < most) {
      compute(t + kTTile > least || miss, t, miss);
      if (odd) poison(t);
    }
    buffer = (buffer + kBuffer) % (kBuffers * kBuffer);
  }

  if (!any) return;
  {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run),
                                                    false, false);
    l_run = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  if (wv + n >= it.v0 + it.nv) return;
  const size_t vr = (size_t)row * bt.H + head;
  const bool all = it.i0 == 0 && it.i1 == it.nt;
  if (PREFIX || (OF == kTallRuns && !all)) {
    float *w, *ml;
    int ml_step;
    const int col = 32 * wave + n;
    if (PREFIX && all) {
      w = whole_at<D>(a.res, bt, 0, vr);
      ml = w + D;
      ml_step = 1;
    } else {
      const int cols = PREFIX ? a.res.cols_pre : a.res.cols_own;
      w = (PREFIX ? a.res.part_pre : a.res.part) +
          (size_t)(2 * run + (it.i0 == 0 ? 1 : 0)) * part_floats<D>(cols);
      ml = w + (size_t)cols * D + col;
      ml_step = cols;
      w += (size_t)col * D;
    }
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(w + 32 * f + 8 * c + 4 * hh) = make_float4(
            acc[f][4 * c], acc[f][4 * c + 1], acc[f][4 * c + 2], acc[f][4 * c + 3]);
    if (hh == 0) {
      ml[0] = m_run;
      ml[ml_step] = l_run;
    }
    return;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;            // (keeps NaN)
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const size_t at = vr * D + 32 * f + 8 * c + 4 * hh;
      const float o0 = acc[f][4 * c] * inv, o1 = acc[f][4 * c + 1] * inv;
      const float o2 = acc[f][4 * c + 2] * inv, o3 = acc[f][4 * c + 3] * inv;
      if (OUT_F32)
        *reinterpret_cast<float4*>(static_cast<float*>(a.O) + at) = make_float4(o0, o1, o2, o3);
      else
        *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.O) + at) =
            make_uint2(pack2_bf16(o0, o1), pack2_bf16(o2, o3));
    }
  if (a.lse && hh == 0) a.lse[vr] = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * kCacheLn2;
  };

  if constexpr (OF == kTallItems) {
    TallItem it;
    if (tall_item(a, block, it)) work(it);
  } else {
    // (sequences by key heads: those that share pages, a prompt's pieces over one context,
    // meet on one XCD, whose L2 they are in)
    const int Wh = walk.total(bt, [&](int before) {
      if (PREFIX || block != 0 || wave != 0 || walk.sb0 + lane >= bt.B) return;
      a.res.meta[(size_t)(walk.sb0 + lane) * kCacheMeta] = before + walk.incl - walk.sb.own;
    });
    const int W = PREFIX ? Wh : Wh * bt.heads_kv;
    const int per = max((W + a.runs - 1) / a.runs, kTLeast);
    if (block == 0 && tid == 0) {
      int32_t* w = a.res.meta + (size_t)bt.B * kCacheMeta;
      if (!PREFIX) w[0] = per;
      w[1] = PREFIX ? per : Wh;
    }
    int u = run * per;
    if (u >= W) return;
    const int end = min(W - u, per) + u;
    while (u < end) {
      int first;
      TallItem it;
      const int at = PREFIX ? 0 : u / Wh * Wh;           // the key head's first tile
      if (!PREFIX && u - at < walk.base) {
        walk.base = 0;
        walk.block(bt, 0);
      }
      const int L = walk.seek(bt, u - at, first);
      first += at;
      it.b = walk.sb0 + L;
      it.r0 = walk.of_lane(walk.sb.s.r0, L);
      int rows, rt, start;
      if constexpr (PREFIX) {
        it.b = walk.sb0 + walk.of_lane(walk.sb.source, L);
        it.hi = walk.of_lane(walk.sb.P, L);
        it.nt = SeqBlock::prefix_tiles(it.hi);
        rows = walk.of_lane(walk.sb.run_rows, L);
        const int rts = SeqBlock::row_tiles(bt, rows, kTRows), step = it.nt + kPrefixStart;
        const int i = (u - first) / step;
        it.hk = i / rts;
        rt = i - it.hk * rts;
        start = first + i * step;
      } else {
        it.s = CacheSeq{it.r0, walk.of_lane(walk.sb.s.n, L), walk.of_lane(walk.sb.s.len, L)};
        rows = it.s.n;
        it.hk = u / Wh;
        start = first;
        for (rt = 0;; ++rt) {
          it.nt = SeqBlock::tall_tiles(bt, it.s.n, it.s.len, rt);
          if (u < start + it.nt + kPrefixStart) break;
          start += it.nt + kPrefixStart;
        }
        it.hi = max(it.s.len - it.s.n + (min((rt + 1) * kTRows, rows * bt.G) - 1) / bt.G + 1, 0);
      }
      it.v0 = rt * kTRows;
      it.nv = min(kTRows, rows * bt.G - it.v0);
      it.i0 = tile_at<kPrefixStart>(u - start, it.nt);
      it.i1 = tile_at<kPrefixStart>(end - start, it.nt);
      u = start + it.nt + kPrefixStart;
      if (it.i0 < it.i1) work(it);
    }
  }
}

}  // namespace skip
