"""The paged cache on the GPU against its float64 oracle: append, attention over the
cache and over listed pages, page selection.

Bounds (u = 2^-24, half a step of float32; 2^-8 half a step of bfloat16, relative):
  rotated rows  the angle is exact to 2^-25 of a turn (2 pi 2^-25 < 4 u in cosine and
      sine), cosine and sine to 2 u more, two products and a sum: 8 u (|x| + |y|)
      before one rounding to bfloat16
  mean keys     float32 sums of n keys as held: n u of the mean of |k|, and the rounding
  logits        sums of d_h products: (d_h + 4) u scale sum |q k| =: delta (base 2, the
      subtraction of the reference: within the 4); a weight is off by 2 delta relative to the
      others, by 4 u for the exponential, by 2^-16 (bf16 output) or 2^-24 for its
      pieces; sums over n tokens add n u: |dO| <= (2 delta + pieces + (2 n + 16) u) sum p |v|,
      and the output's rounding; |dLSE| <= delta + (n + 16) u + u |LSE|
"""
import sys

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    from paper_2607_25422_amd import binding
    return binding


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=np.int32))).cuda()


class Setup:
    """seqs: (new tokens, tokens held) of every sequence, pages in any order.  The pool's
    slots that hold no token are NaN, or `stale`."""

    def __init__(self, B, seqs, H=8, hk=2, D=64, page=32, seed=0, dtype="bf16", o_f32=False,
                 scale=None, extra_rows=0, stale=float("nan"), shared=(), mean=True, rows=None):
        rng = np.random.default_rng(seed)
        self.B, self.H, self.hk, self.D, self.page, self.seqs = B, H, hk, D, page, seqs
        self.ro = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.lens = np.array([ln for _, ln in seqs], dtype=np.int32)
        need = [-(-ln // page) for _, ln in seqs]
        pages = sum(need) + 2
        order = rng.permutation(pages)
        self.table = np.full((len(seqs), max(max(need), 1) + 1), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        K = torch.from_numpy(rng.standard_normal((pages, hk, page, D))).bfloat16()
        V = torch.from_numpy(rng.standard_normal((pages, hk, page, D))).bfloat16()
        for a, b, t in shared:              # sequence b's first t tokens are sequence a's
            for j in range(-(-t // page)):
                n = min(page, t - j * page)
                if n == page:
                    self.table[b, j] = self.table[a, j]
                else:
                    K[self.table[b, j], :, :n] = K[self.table[a, j], :, :n]
                    V[self.table[b, j], :, :n] = V[self.table[a, j], :, :n]
        held = np.zeros((pages, page), dtype=bool)
        for b, (_, ln) in enumerate(seqs):
            for t in range(ln):
                held[self.table[b, t // page], t % page] = True
        K.transpose(1, 2)[~torch.from_numpy(held)] = stale
        V.transpose(1, 2)[~torch.from_numpy(held)] = stale
        m = torch.from_numpy(rng.standard_normal((pages, hk, D))).bfloat16() if mean else None
        total = int(self.ro[-1]) + extra_rows
        self.p = B.make_problem(dtype, B=len(seqs), d=H * D, H=H, d_h=D,
                                kept_offsets=self.ro, sm_scale=scale, o_f32=o_f32)
        self.p.total_kept = total
        self.p.k_max = max(self.p.k_max, -(-total // len(seqs)))
        self.p.L_max = int(self.lens.max(initial=0))
        self.scale = float(self.p.sm_scale)
        self.cache = B.KvCache(K.cuda(), V.cuda(), None if m is None else m.cuda(), dev(self.table))
        self.row_offsets, self.dlens = dev(self.ro), dev(self.lens)
        q = torch.from_numpy(rng.standard_normal((total, H, D)))
        self.q = q.bfloat16().cuda()
        self.rng = rng

    def new_rows(self, packed):
        dt = torch.float32 if self.p.dtype == 0 else torch.bfloat16
        H, hk, D, M = self.H, self.hk, self.D, self.p.total_kept
        x = torch.from_numpy(self.rng.standard_normal((M, (H + 2 * hk) * D + 24))).to(dt).cuda()
        cut = [x[:, :H * D], x[:, H * D:(H + hk) * D], x[:, (H + hk) * D:(H + 2 * hk) * D]]
        if not packed:
            cut = [c.contiguous() for c in cut]
        return [c.unflatten(1, (-1, D)) for c in cut]

    def reference(self, listed=None):
        c = self.cache
        return co.attention(f64(self.q), f64(c.k), f64(c.v), self.table, self.ro, self.lens,
                            self.scale, listed)

    def bounds(self, ref, o_f32):
        O, lse, A = ref
        n = max(int(self.lens.max()), 1)
        k = f64(self.cache.k)
        delta = (self.D + 4) * U * abs(self.scale) * np.abs(f64(self.q)).sum(-1).max(-1)[:, None]
        delta = delta * np.nanmax(np.where(np.isfinite(k), np.abs(k), 0)) + np.zeros_like(lse)
        rel = 2 * delta + (2.0 ** -24 if o_f32 else 2.0 ** -16) + (2 * n + 16) * U
        return (rel[..., None] * A + (U if o_f32 else BF) * np.abs(O),
                delta + (n + 16) * U + U * np.abs(np.where(np.isfinite(lse), lse, 0)))

    def check(self, got, ref, o_f32, rows=None):
        r = slice(0, int(self.ro[-1])) if rows is None else rows
        tolO, tolL = self.bounds(ref, o_f32)
        O, lse = f64(got[0])[r], f64(got[1])[r]
        none = ref[1][r] == -np.inf
        assert (lse[none] == -np.inf).all() and (O[none] == 0).all()
        dO = np.abs(O - ref[0][r]) - tolO[r]
        dL = np.abs(lse[~none] - ref[1][r][~none]) - tolL[r][~none]
        worst = float(dO.max(initial=-1)), float(dL.max(initial=-1))
        assert bool(np.isfinite(O).all()) and bool(np.isfinite(lse[~none]).all()), worst
        assert max(worst) <= 0, worst


def attn(s, B, **kw):
    return B.cache_attn(s.p, s.cache, s.q, s.row_offsets, s.dlens, **kw)


# ---------------------------------------------------------------------------
# Append

FREQ = lambda n: np.float32(10000.0) ** (-np.arange(n, dtype=np.float32) / max(n, 1))

APPEND = [
    dict(seqs=[(1, 1)]),
    dict(seqs=[(1, 32), (1, 33), (2, 34), (0, 5), (1, 64)], dtype="f32"),
    dict(seqs=[(70, 75), (33, 33), (1, 200)], D=128, H=6, hk=3, page=64, packed=False),
    dict(seqs=[(130, 300), (3, 259)], D=128, H=4, hk=4, page=128, style="pairs", dtype="f32"),
    dict(seqs=[(300, 513), (1, 256), (0, 0), (5, 5)], page=256, dims=32, positions=True),
    dict(seqs=[(1, 40 + i) for i in range(70)], H=16, hk=1, dims=48, style="pairs"),
    dict(seqs=[(3, 35)] * 65, dims=16),
    dict(seqs=[(9, 20), (1, 64)], dims=0),
    dict(seqs=[(2, 50), (7, 90)], mean=False, q=False),
    dict(seqs=[(40, 100), (3, 3)], extra_rows=11),
    dict(seqs=[(50, 80), (34, 40), (0, 3), (1, 64)], H=9, hk=1, page=64, dims=32, dtype="f32"),
]


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(B, case):
    c = dict(APPEND[case])
    style, dims = c.pop("style", "halves"), c.pop("dims", None)
    positions, packed, with_q = c.pop("positions", False), c.pop("packed", True), c.pop("q", True)
    s = Setup(B, seed=case, **c)
    q, k, v = s.new_rows(packed)
    dims = s.D if dims is None else dims
    freq, M = FREQ(dims // 2), int(s.ro[-1])
    pos = s.rng.integers(0, 2_000_000, s.p.total_kept).astype(np.int32)   # far ones, too
    K0, V0 = s.cache.k.clone(), s.cache.v.clone()
    m0 = None if s.cache.mean is None else s.cache.mean.clone()
    out = torch.full((s.p.total_kept, s.H, s.D), 7.0, dtype=torch.bfloat16, device="cuda")
    say("[append]", case, c)
    rot = B.Rotation(torch.from_numpy(freq).cuda(), style) if dims else None
    B.cache_append(s.p, s.cache, q if with_q else None, k, v, s.row_offsets, s.dlens, rotation=rot,
                   positions=dev(pos) if positions else None, out=out if with_q else None)
    torch.cuda.synchronize()
    tok = np.concatenate([co.tokens(s.ro, s.lens, b) for b in range(len(s.seqs))])
    at = pos[:M] if positions else tok

    def close(got, x):
        x = f64(x)[:M]
        want = co.rotate(x, at, freq.astype(np.float64), style)
        size = co.rotate(np.abs(x), np.zeros(M), freq, style)
        r = dims // 2
        part = size.copy()
        if dims and style == "halves":
            part[..., :r], part[..., r:dims] = size[..., r:dims], size[..., :r]
        elif dims:
            part[..., 0:dims:2], part[..., 1:dims:2] = size[..., 1:dims:2], size[..., 0:dims:2]
        tol = BF * np.abs(want) + (1 + BF) * 8 * U * (size + part)
        assert (np.abs(got - want) <= tol).all()
    if with_q:
        close(f64(out)[:M], q)
        assert (out[M:] == 7).all()
    # the cache: what was written, and nothing else
    K1, V1 = s.cache.k, s.cache.v
    seq = np.concatenate([[b] * n for b, (n, _) in enumerate(s.seqs)]).astype(int)
    pg = torch.from_numpy(s.table[seq, tok // s.page].astype(np.int64)).cuda()
    slot = torch.from_numpy(tok % s.page).cuda()
    close(f64(K1[pg, :, slot]), k)
    assert torch.equal(V1[pg, :, slot], v[:M].bfloat16())
    K0[pg, :, slot], V0[pg, :, slot] = K1[pg, :, slot], V1[pg, :, slot]
    assert torch.equal(K0.view(torch.int16), K1.view(torch.int16))
    assert torch.equal(V0.view(torch.int16), V1.view(torch.int16))
    if m0 is None:
        return
    for b, (n, ln) in enumerate(s.seqs):
        for j in range((ln - n) // s.page, -(-ln // s.page)) if n else ():
            e = min(s.page, ln - j * s.page)
            keys = f64(K1[int(s.table[b, j]), :, :e])
            want, got = keys.mean(1), f64(s.cache.mean[int(s.table[b, j])])
            tol = BF * np.abs(want) + (1 + BF) * (e + 2) * U * np.abs(keys).mean(1)
            assert (np.abs(got - want) <= tol).all(), (b, j)
            m0[int(s.table[b, j])] = s.cache.mean[int(s.table[b, j])]
    assert torch.equal(m0.view(torch.int16), s.cache.mean.view(torch.int16))


def test_append_again_after_a_cut(B):
    """A sequence cut back and appended to again: the cache, means among it, as if the
    cut tokens had never been."""
    s = Setup(B, [(40, 70)])
    q, k, v = s.new_rows(True)
    rot = B.Rotation(torch.from_numpy(FREQ(32)).cuda())
    B.cache_append(s.p, s.cache, q, k, v, s.row_offsets, s.dlens, rotation=rot)
    B.cache_append(s.p, s.cache, q, -k, v, s.row_offsets, dev([60]), rotation=rot)
    again = [x.clone() for x in (s.cache.k, s.cache.v, s.cache.mean)]
    t = Setup(B, [(40, 70)])
    q, k, v = t.new_rows(True)
    t.cache.k[:], t.cache.v[:] = 0, 0
    B.cache_append(t.p, t.cache, q, -k, v, t.row_offsets, dev([60]), rotation=rot)
    for j in (0, 1):
        e = min(32, 60 - 32 * j)
        pg = int(t.table[0, j])
        for a, x in zip(again, (t.cache.k, t.cache.v)):
            new = slice(max(0, 20 - 32 * j), e)
            assert torch.equal(a[pg, :, new], x[pg, :, new])
    keys = f64(again[0][int(s.table[0, 1]), :, :28])
    tol = BF * np.abs(keys.mean(1)) + (1 + BF) * 30 * U * np.abs(keys).mean(1)
    assert (np.abs(f64(again[2][int(s.table[0, 1])]) - keys.mean(1)) <= tol).all()


def test_append_without_a_page(B):
    """Tokens whose page is missing are not written; the others are."""
    s = Setup(B, [(40, 70), (2, 3)])
    q, k, v = s.new_rows(True)
    table = s.table.copy()
    table[0, 1], table[0, 2] = -1, 1 << 20
    cache = B.KvCache(s.cache.k.clone(), s.cache.v.clone(), s.cache.mean.clone(), dev(table))
    out = B.cache_append(s.p, cache, q, k, v, s.row_offsets, s.dlens)
    torch.cuda.synchronize()
    assert torch.equal(out, q.bfloat16())
    for a, b in ((cache.k, s.cache.k), (cache.v, s.cache.v)):
        for pg in range(a.shape[0]):
            if pg not in (table[0, 0], table[1, 0]):
                assert torch.equal(a[pg].view(torch.int16), b[pg].view(torch.int16))
    assert torch.equal(cache.v[int(table[1, 0]), :, 1:3].transpose(0, 1), v[40:42])


@pytest.mark.parametrize("page,n", [(32, 9), (64, 50), (256, 300)])
def test_append_of_more_rows_than_tokens(B, page, n):
    """Rows before their sequence's first token: their queries are left, nothing of them
    is written; the others as if they were alone."""
    s = Setup(B, [(n, n), (n, n), (2, 2)], page=page, D=64, seed=23)
    lens = np.array([n - 5, 0, 2], np.int32)
    q, k, v = s.new_rows(True)
    rot = B.Rotation(torch.from_numpy(FREQ(32)).cuda())
    out = torch.full((s.p.total_kept, s.H, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    one = [x.clone() for x in (s.cache.k, s.cache.v, s.cache.mean)]
    B.cache_append(s.p, s.cache, q, k, v, s.row_offsets, dev(lens), rotation=rot, out=out)
    torch.cuda.synchronize()
    lost = [*range(5), *range(n, 2 * n)]
    held = [*range(5, n), 2 * n, 2 * n + 1]
    assert (out[lost] == 7).all()
    p = B.make_problem("bf16", B=3, d=s.H * 64, H=s.H, d_h=64, kept_offsets=[0, n - 5, n - 5, n - 3])
    p.L_max = n
    cache = B.KvCache(*one, s.cache.page_table)
    want = B.cache_append(p, cache, *(x[held].contiguous() for x in (q, k, v)),
                          dev([0, n - 5, n - 5, n - 3]), dev(lens), rotation=rot)
    torch.cuda.synchronize()
    assert torch.equal(out[held], want)
    for a, b in zip((s.cache.k, s.cache.v, s.cache.mean), one):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


# ---------------------------------------------------------------------------
# Attention

ATTN = [
    dict(seqs=[(1, 1)]),
    dict(seqs=[(1, 31), (1, 32), (1, 33), (1, 0), (0, 9), (1, 512)], D=128),
    dict(seqs=[(1, 1300), (1, 5), (1, 700), (2, 64)], D=128, page=64),            # parts
    dict(seqs=[(1, 4097)], H=16, hk=1, page=128, o_f32=True),
    dict(seqs=[(1, 900), (1, 1), (0, 0), (1, 513)], H=32, hk=1, D=128, page=256),
    dict(seqs=[(5, 600), (3, 3), (8, 40)], H=12, hk=3),                           # two blocks
    dict(seqs=[(40, 40), (65, 700), (1, 530)], H=8, hk=4, D=128, o_f32=True),     # four
    dict(seqs=[(130, 131)], H=5, hk=5, page=64),
    dict(seqs=[(33, 20), (2, 600)], H=4, hk=2),                # more rows than tokens held
    dict(seqs=[(1 + i % 2, 20 + 37 * (i % 17)) for i in range(130)], H=4, hk=2),
    dict(seqs=[(1, 700), (3, 800)], scale=-0.3, D=128),
    dict(seqs=[(1, 700), (3, 90)], scale=0.0),
    dict(seqs=[(1, 700), (3, 90)], extra_rows=9),
    dict(seqs=[(200, 200), (300, 777), (129, 1500)], H=8, hk=2, D=128, page=64),
    dict(seqs=[(257, 257), (0, 50), (64, 64), (1, 900)], H=3, hk=1, D=64, o_f32=True),
    dict(seqs=[(257, 300), (130, 700), (1, 64)], H=3, hk=1, D=128, page=256),     # taken whole
    dict(seqs=[(40, 41)] * 90, H=32, hk=32, D=64, page=32),                       # 90 items a head
    dict(seqs=[(9, 2000), (5, 1000)], H=16, hk=2, D=128, page=32, extra_rows=5, o_f32=True),
    # runs over more than 64 sequences, key head by key head
    dict(seqs=[(33 + 3 * (i % 40), 300 + 61 * (i % 13)) for i in range(70)], H=3, hk=3, D=64),
    dict(seqs=[(20 * (i % 3), 790 + i) for i in range(131)], H=6, hk=2, D=128, page=64, o_f32=True),
]


@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(B, case):
    c = ATTN[case]
    s = Setup(B, seed=100 + case, **c)
    say("[attn]", case, c)
    f32 = c.get("o_f32", False)
    out = (torch.full((s.p.total_kept, s.H, s.D), 7.0, device="cuda",
                      dtype=torch.float32 if f32 else torch.bfloat16),
           torch.full((s.p.total_kept, s.H), 7.0, device="cuda"))
    attn(s, B, out=out)
    torch.cuda.synchronize()
    s.check(out, s.reference(), f32)
    M = int(s.ro[-1])
    assert (out[0][M:] == 7).all() and (out[1][M:] == 7).all()       # left as they were
    O2, lse2 = attn(s, B, out=(torch.empty_like(out[0]), None))
    torch.cuda.synchronize()
    assert lse2 is None and torch.equal(O2[:M], out[0][:M])


# (sequences whose keys and values are 64 MB or more, where prefixes are items of their
# own, and one batch of fewer)
SHARED = [
    dict(seqs=[(1, 2140), (1, 2800), (1, 2101), (1, 2333), (1, 2102), (1, 2164)],
         shared=[(0, i, 2100) for i in range(1, 6)], ids=[0] * 6, P=[2100] * 6, H=16, hk=8, D=128),
    dict(seqs=[(2, 2900), (1, 2145), (4, 2200), (1, 40), (1, 2300), (0, 2250)],
         shared=[(0, 1, 2113), (3, 4, 32), (3, 5, 32)], ids=[5, 5, -1, 2, 2, 2],
         P=[2113, 2113, 2113, 32, 32, 32], H=16, hk=8, D=128, page=64),
    # new tokens inside the prefix, a prefix that some sequences have not reached
    dict(seqs=[(12, 5590), (10, 5585), (3, 5100)], shared=[(0, 1, 5580), (0, 2, 5100)], ids=[1] * 3,
         P=[5580] * 3, H=16, hk=8, D=128, page=256, o_f32=True),
    # a run across blocks of 64 sequences and of 128 virtual rows, alone ones between
    dict(seqs=[(1, 1320 + i % 9) for i in range(100)],
         shared=[(0, i, 1310) for i in range(1, 70)] + [(72, i, 1280) for i in range(73, 100)],
         ids=[0] * 70 + [1, 3] + [2] * 28, P=[1310] * 70 + [1310, 1310] + [1280] * 28, H=8, hk=2),
    # ids equal, lengths not: not shared
    dict(seqs=[(1, 8300), (1, 8200)], ids=[0, 0], P=[64, 96], shared=[], H=8, hk=8, D=128),
    # 16 query heads a key head, two tokens: two blocks of 16; float32 output
    dict(seqs=[(2, 8500 + 300 * i) for i in range(9)], shared=[(0, i, 8400) for i in range(1, 9)],
         ids=[7] * 9, P=[8400] * 9, H=48, hk=3, D=64, page=128, o_f32=True, extra_rows=2),
    dict(seqs=[(1, 640), (1, 700), (1, 601)], shared=[(0, 1, 600), (0, 2, 600)], ids=[0, 0, 0],
         P=[600, 600, 600]),
]


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_shared_prefixes(B, case):
    c = dict(SHARED[case])
    ids, P = c.pop("ids"), c.pop("P")
    s = Setup(B, seed=200 + case, **c)
    say("[shared]", case)
    whole = 4 * len(ids) * s.hk * int(s.lens.max()) * s.D
    assert (whole >= 64 << 20) == (case != len(SHARED) - 1)
    got = attn(s, B, prefix_ids=dev(ids), prefix_lens=dev(P))
    torch.cuda.synchronize()
    ref = s.reference()
    s.check(got, ref, c.get("o_f32", False))
    s.check(attn(s, B), ref, c.get("o_f32", False))


def test_prefixes_of_sequences_that_are_passed_over(B):
    """A run's sequences without rows, its first one among them, need no pages; one that
    has fewer tokens than the prefix reads its own."""
    ids, P = [4] * 8, [2100] * 8
    s = Setup(B, [(0, 0), (1, 2140), (0, 0), (2, 2800), (1, 2101), (1, 900), (1, 2333), (0, 0)],
              shared=[(1, i, 2100) for i in (3, 4, 6)], H=16, hk=8, D=128, seed=211)
    say("[passed over]")
    assert (s.table[[0, 2, 7]] == -1).all() and 4 * 8 * 8 * 2800 * 128 >= 64 << 20
    got = attn(s, B, prefix_ids=dev(ids), prefix_lens=dev(P))
    torch.cuda.synchronize()
    s.check(got, s.reference(), False)


def test_prefixes_longer_than_any_sequence(B):
    """prefix_lens past L_max: no sequence holds such a prefix, all read their own."""
    s = Setup(B, [(1, 5600), (2, 5600), (1, 5590), (1, 5600)], H=16, hk=8, D=128, page=32, seed=15)
    assert 4 * 4 * 8 * 5600 * 128 >= 64 << 20
    ref = s.reference()
    for P in ([6000, 6000, 6000, 6000], [6000, 7000, 7000, 9000], [2 ** 31 - 1] * 4):
        got = attn(s, B, prefix_ids=dev([0] * 4), prefix_lens=dev(P))
        torch.cuda.synchronize()
        s.check(got, ref, False)


@pytest.mark.parametrize("o_f32", [False, True])
@pytest.mark.parametrize("n,ln", [(40, 40), (7, 600), (200, 200), (40, 700)])
def test_what_a_row_does_not_see_does_not_reach_it(B, n, ln, o_f32):
    """Infinities and NaN in the keys and values of later new tokens: rows before them
    are as without, rows after them are not finite where they meet them (infinity or
    NaN: what is not finite is found apart from the products)."""
    s = Setup(B, [(n, ln), (n, ln)], H=4, hk=2, D=128, page=64, o_f32=o_f32, seed=9)
    ref = s.reference()
    for b, bad in ((0, n - 3), (1, n // 2)):
        t = ln - n + bad
        pg = int(s.table[b, t // 64])
        s.cache.v[pg, 0, t % 64, 5] = float("inf")
        s.cache.v[pg, 1, t % 64, 77] = float("nan")
        s.cache.k[pg, 1, t % 64, 3] = float("nan")
    got = attn(s, B)
    torch.cuda.synchronize()
    for b, bad in ((0, n - 3), (1, n // 2)):
        s.check(got, ref, o_f32, rows=slice(b * n, b * n + bad))
        after = got[0][b * n + bad:(b + 1) * n].float()
        assert not torch.isfinite(after[:, :2, 5]).any() and torch.isnan(after[:, 2:]).all()
        assert torch.isfinite(after[:, :2, :5]).all() and torch.isfinite(after[:, :2, 6:]).all()


def plant(s, tokens):
    """An infinity and NaN in the values, NaN in the keys, of one token of some
    sequences."""
    for b, t in tokens:
        pg, at = int(s.table[b, t // s.page]), t % s.page
        s.cache.v[pg, 0, at, 5] = float("inf")
        s.cache.v[pg, 1, at, s.D - 3] = float("nan")
        s.cache.k[pg, 1, at, 3] = float("nan")


def check_planted(s, got, ref, o_f32, b, t):
    """The sequence's rows before token t are as without; the others are not finite
    where they meet it."""
    r0, n, ln, G = int(s.ro[b]), *s.seqs[b], s.H // s.hk
    first = r0 + min(max(t - (ln - n), 0), n)
    s.check(got, ref, o_f32, rows=slice(r0, first))
    after = got[0][first:r0 + n].float()
    assert not torch.isfinite(after[:, :G, 5]).any() and torch.isnan(after[:, G:2 * G]).all()
    assert torch.isfinite(after[:, :G, :5]).all() and torch.isfinite(after[:, :G, 6:]).all()
    assert torch.isfinite(after[:, 2 * G:]).all()


@pytest.mark.parametrize("n,ln,page,D,o_f32", [
    (130, 1500, 32, 64, True), (130, 1500, 64, 128, False), (300, 300, 256, 64, False),
    (5, 400, 32, 64, True), (9, 1800, 128, 128, False)])
def test_every_form_keeps_unseen_values_out(B, n, ln, page, D, o_f32):
    """Rows in runs and whole, both head sizes, few and many new tokens."""
    s = Setup(B, [(n, ln), (n, ln), (1, ln)], H=6, hk=3, D=D, page=page, o_f32=o_f32, seed=10)
    ref = s.reference()
    at = [(0, ln - 2), (1, ln - n // 2 - 1)]
    plant(s, at)
    got = attn(s, B)
    torch.cuda.synchronize()
    for b, t in at:
        check_planted(s, got, ref, o_f32, b, t)
    s.check(got, ref, o_f32, rows=slice(2 * n, 2 * n + 1))


def test_unseen_values_inside_a_shared_prefix(B):
    """New tokens inside the prefix, which not all rows of the run see."""
    s = Setup(B, [(12, 5606), (10, 5601), (16, 5616)], shared=[(0, 1, 5600), (0, 2, 5600)], H=16,
              hk=8, D=128, page=32, seed=12)
    assert 4 * 3 * 8 * 5616 * 128 >= 64 << 20
    ref = s.reference()
    plant(s, [(0, 5597)])
    got = attn(s, B, prefix_ids=dev([0] * 3), prefix_lens=dev([5600] * 3))
    torch.cuda.synchronize()
    for b in range(3):
        check_planted(s, got, ref, False, b, 5597)


@pytest.mark.parametrize("n,ln,page,D", [(2, 300, 32, 64), (70, 600, 32, 128), (70, 600, 64, 64),
                                         (70, 1700, 32, 64), (70, 1700, 128, 128)])
def test_missing_pages_in_every_form(B, n, ln, page, D):
    s = Setup(B, [(n, ln), (n, ln - 90)], H=4, hk=2, D=D, page=page, seed=13)
    last = (ln - 1) // page
    s.table[0, 1], s.table[0, last], s.table[1, 0] = -1, -9, 1 << 30
    s.cache.page_table.copy_(dev(s.table))
    got = attn(s, B)
    torch.cuda.synchronize()
    s.check(got, s.reference(), False)
    listed = np.tile(np.arange(min(last + 1, 12), dtype=np.int32), (2 * n, 2, 1))
    got = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, dev(listed))
    torch.cuda.synchronize()
    s.check(got, s.reference(listed), False)


def test_pages_that_a_whole_run_misses(B):
    """A prefix's page that is in none of its sequences' tables."""
    s = Setup(B, [(1, 2900), (2, 2700), (1, 2600)] * 2, H=16, hk=8, D=128, page=32, seed=14,
              shared=[(0, i, 2500) for i in range(1, 6)])
    assert 4 * 6 * 8 * 2900 * 128 >= 64 << 20
    s.table[:, 3] = s.table[:, 40] = -1
    s.cache.page_table.copy_(dev(s.table))
    got = attn(s, B, prefix_ids=dev([0] * 6), prefix_lens=dev([2500] * 6))
    torch.cuda.synchronize()
    s.check(got, s.reference(), False)


def test_large_values_and_logits(B):
    """Values near the largest bfloat16 keep their sums finite; logits far apart."""
    s = Setup(B, [(1, 3000), (2, 70)], H=4, hk=2, seed=3, scale=40.0, o_f32=True)
    s.cache.v[:] = torch.where(torch.isfinite(s.cache.v), 3.3e38, s.cache.v)
    got = attn(s, B)
    torch.cuda.synchronize()
    s.check(got, s.reference(), True)


@pytest.mark.parametrize("n,ln,page,D,o_f32", [
    (1, 200, 32, 64, False), (3, 1300, 64, 128, False), (40, 300, 32, 64, True),
    (130, 1500, 64, 128, False), (1, 4000, 32, 64, True), (10, 900, 32, 128, False),
    (12, 300, 64, 64, True)])
def test_logits_past_float32(B, n, ln, page, D, o_f32):
    """A finite product whose scaled value is not: below float32 it weighs nothing, above
    it the row is not finite (a row of zeros would be one that sees no token).  The rows
    looked at have logits of 2^63 and more otherwise, so that the largest alone has a
    weight: their results are its value."""
    s = Setup(B, [(n, ln), (n, ln)], H=4, hk=2, D=D, page=page, o_f32=o_f32, scale=8.0, seed=16)
    big = 2.0 ** 60
    for b in range(2):
        s.cache.k[int(s.table[b, 0]), :, 5] = big          # (times the query: 2^126 or 2^127)
        s.q[(b + 1) * n - 1] = big if b == 0 else -big
    k = np.abs(f64(s.cache.k))
    tol = (D + 4) * U * s.scale * big * np.where(k < big, k, 0.0).sum(-1).max()
    got = attn(s, B)
    listed = np.tile(np.arange(12, dtype=np.int32), (2 * n, 2, 1))
    by = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, dev(listed))
    torch.cuda.synchronize()
    for (O, lse), ref in ((got, s.reference()), (by, s.reference(listed))):
        assert not torch.isfinite(O[n - 1].float()).any() and not torch.isfinite(lse[n - 1]).any()
        assert (f64(O)[2 * n - 1] == ref[0][2 * n - 1]).all()
        want = ref[1][2 * n - 1]
        assert (np.abs(f64(lse)[2 * n - 1] - want) <= tol + 4 * U * np.abs(want)).all()
        others = [r for r in range(2 * n) if r not in (n - 1, 2 * n - 1)]
        assert torch.isfinite(O[others].float()).all() and torch.isfinite(lse[others]).all()


def test_logits_past_float32_in_a_shared_prefix(B):
    """As above, for rows of one prefix item: the rows of the first sequence are not
    finite, those of the second have one weight, those of the third are as ever."""
    s = Setup(B, [(2, 5610), (1, 5620), (1, 5605)], shared=[(0, 1, 5600), (0, 2, 5600)], H=16,
              hk=8, D=128, page=64, scale=8.0, seed=24)
    assert 4 * 3 * 8 * 5620 * 128 >= 64 << 20
    big = 2.0 ** 60
    s.cache.k[int(s.table[0, 43]), :, 11] = big
    s.q[:2], s.q[2] = big, -big
    s.q[3] = s.q[3].abs() * -0.5                    # (its logit of that token: far below the others)
    ref = s.reference()
    O, lse = attn(s, B, prefix_ids=dev([0] * 3), prefix_lens=dev([5600] * 3))
    torch.cuda.synchronize()
    assert not torch.isfinite(O[:2].float()).any() and not torch.isfinite(lse[:2]).any()
    assert (f64(O)[2] == ref[0][2]).all()
    k = f64(s.cache.k)
    delta = (128 + 4) * U * 8 * np.abs(f64(s.q[3])).sum(-1).max() * np.nanmax(np.where(k < big, np.abs(k), 0))
    rel = 2 * delta + 2.0 ** -16 + (2 * 5620 + 16) * U
    assert (np.abs(f64(O)[3] - ref[0][3]) <= rel * ref[2][3] + BF * np.abs(ref[0][3])).all()


def test_missing_pages_are_passed_over(B):
    s = Setup(B, [(1, 700), (3, 90)], seed=4)
    s.table[0, 3], s.table[0, 20], s.table[1, 0] = -1, 1 << 29, -5
    s.cache.page_table.copy_(dev(s.table))
    got = attn(s, B)
    torch.cuda.synchronize()
    s.check(got, s.reference(), False)


def test_offsets_past_32_bits(B):
    """Pages at more than 2^31 elements into the pool."""
    hk, page, D = 8, 256, 128
    pages = (1 << 31) // (hk * page * D) + 3
    cache = B.new_kv_cache(pages, hk, page, D, dev([[pages - 1, pages - 3, 1]]))
    p = B.make_problem("bf16", B=1, d=8 * D, H=8, d_h=D, kept_offsets=[0, 260])
    p.L_max = 600
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(260, h, D, generator=g, device="cuda").bfloat16() for h in (8, hk, hk))
    ro, lens = dev([0, 260]), dev([260])
    qr = B.cache_append(p, cache, q, k, v, ro, lens)
    got = attn_out = B.cache_attn(p, cache, qr, ro, lens)
    sel = B.cache_select(p, cache, qr, ro, lens, 2)
    by = B.cache_attn_pages(p, cache, qr, ro, lens, sel)
    torch.cuda.synchronize()
    small = B.KvCache(torch.stack([cache.k[pages - 1], cache.k[pages - 3]]),
                      torch.stack([cache.v[pages - 1], cache.v[pages - 3]]), None, dev([[0, 1, -1]]))
    for a, b in zip(B.cache_attn(p, small, qr, ro, lens), got):
        assert torch.equal(a, b)
    for a, b in zip(B.cache_attn_pages(p, small, qr, ro, lens, sel), by):
        assert torch.equal(a, b)
    assert sel[-1].tolist() == [[0, 1]] * hk and sel[0].tolist() == [[0, -1]] * hk


# ---------------------------------------------------------------------------
# Selection and attention over pages

SELECT = [
    dict(seqs=[(1, 1)], n_sel=3),
    dict(seqs=[(1, 2000), (3, 700), (1, 0), (0, 50), (1, 96)], n_sel=9, n_first=1, n_last=2),
    dict(seqs=[(1, 5000)], H=16, hk=2, D=128, n_sel=40, n_first=0),
    dict(seqs=[(2, 40000)], H=2, hk=1, n_sel=64, n_last=3),                 # 1250 pages
    dict(seqs=[(20, 300), (70, 400)], H=32, hk=1, D=128, page=64, n_sel=4, extra_rows=3),
    dict(seqs=[(1, 3000)], n_sel=200),
    dict(seqs=[(1, 600 + 50 * (i % 5)) for i in range(70)], H=6, hk=3, n_sel=5),
    dict(seqs=[(4, 1500), (1, 900)], H=24, hk=1, D=128, page=128, n_sel=6, o_f32=True),
    dict(seqs=[(1, 80000), (1, 40)], H=2, hk=1, n_sel=30, n_last=2),        # 2500 pages, few rows
    dict(seqs=[(130, 66000)], H=2, hk=2, n_sel=3),                          # and many
    dict(seqs=[(70, 300), (1, 20)], H=32, hk=16, D=128, n_sel=5, o_f32=True),     # a wave each
    dict(seqs=[(200, 300), (150, 260)], H=6, hk=3, n_sel=5),                      # likewise
    dict(seqs=[(530, 600)], H=4, hk=2, D=128, n_sel=4, extra_rows=2),
]


@pytest.mark.parametrize("case", range(len(SELECT)))
def test_selected_pages(B, case):
    c = dict(SELECT[case])
    n_sel, nf, nl = c.pop("n_sel"), c.pop("n_first", 1), c.pop("n_last", 1)
    s = Setup(B, seed=300 + case, **c)
    say("[pages]", case, c)
    out = torch.full((s.p.total_kept, s.hk, n_sel), -9, dtype=torch.int32, device="cuda")
    B.cache_select(s.p, s.cache, s.q, s.row_offsets, s.dlens, n_sel, nf, nl, out=out)
    torch.cuda.synchronize()
    M = int(s.ro[-1])
    want = co.select(f64(s.q), f64(s.cache.mean), s.table, s.page, s.ro, s.lens, n_sel, nf, nl)
    assert (out.cpu().numpy()[:M] == want[:M]).all()
    assert (out[M:] == -9).all()
    got = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, out)
    torch.cuda.synchronize()
    s.check(got, s.reference(want), c.get("o_f32", False))


def test_ties_take_the_lower_page(B):
    s = Setup(B, [(1, 1600), (1, 1600)], page=32, seed=5)
    s.cache.mean[:] = 1.0
    out = B.cache_select(s.p, s.cache, s.q, s.row_offsets, s.dlens, 7, 0, 2)
    assert out[0, 0].tolist() == [0, 1, 2, 3, 4, 48, 49] and (out == out[0, 0]).all()


def test_listed_pages_as_they_are_given(B):
    """Any order, the same page twice, entries outside the row's pages, none at all."""
    s = Setup(B, [(1, 1000), (2, 200), (1, 300)], seed=6, page=32)
    listed = np.full((4, 2, 19), -1, dtype=np.int32)
    listed[0, 0] = s.rng.permutation(40)[:19]            # 32 pages: some are behind the row
    listed[0, 1] = [3, 3, 1, 30, 3] + [-7] * 14
    listed[1, :, 5] = 6
    listed[2] = s.rng.integers(-2, 9, (2, 19))
    got = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, dev(listed))
    torch.cuda.synchronize()
    s.check(got, s.reference(listed), False)


@pytest.mark.parametrize("G,hk,n,D,page,o_f32", [
    (17, 2, 530, 64, 32, False), (32, 2, 520, 128, 64, False), (20, 16, 70, 64, 32, True),
    (25, 3, 350, 128, 32, True)])
def test_a_wave_an_item_of_two_row_blocks(B, G, hk, n, D, page, o_f32):
    """1024 rows and key heads or more, 17 to 32 query heads on one, listed pages that end
    inside the row's own, and none."""
    s = Setup(B, [(n, n + 5)], H=G * hk, hk=hk, D=D, page=page, o_f32=o_f32, seed=20)
    assert n * hk >= 1024 and 16 < G <= 32
    listed = s.rng.integers(-1, -(-(n + 5) // page) + 1, (n, hk, 3)).astype(np.int32)
    listed[n // 2, 0] = -1
    got = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, dev(listed))
    torch.cuda.synchronize()
    s.check(got, s.reference(listed), o_f32)


@pytest.mark.parametrize("seqs,n_sel", [([(40, 40)] * 1650, 17), ([(1, 32 * 16384 + 9), (2, 70)], 30)])
def test_listed_pages_past_the_selections_limits(B, seqs, n_sel):
    """More than 65535 rows, more than 16384 pages a sequence; the call's own workspace."""
    s = Setup(B, seqs, H=1, hk=1, seed=19)
    rows = s.p.total_kept
    assert rows > 65535 or s.p.L_max > 32 * 16384
    listed = np.full((rows, 1, n_sel), -1, dtype=np.int32)
    top = max(-(-int(s.lens.max()) // 32), n_sel)
    listed[:, 0, ::3] = s.rng.integers(0, top, (rows, len(range(0, n_sel, 3))))
    listed[:, 0, 0] = 0
    listed[0, 0, -1] = (seqs[0][1] - 1) // 32
    got = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, dev(listed))
    torch.cuda.synchronize()
    s.check(got, s.reference(listed), False)
    with pytest.raises(B.SkipError):
        B.cache_select(s.p, s.cache, s.q, s.row_offsets, s.dlens, n_sel)


@pytest.mark.parametrize("H,hk,D,seqs", [
    (96, 8, 128, [(1, 700), (2, 40), (0, 9)]), (130, 130, 64, [(1, 70), (3, 900)]),
    (160, 8, 128, [(20, 800), (1, 33)]), (640, 20, 64, [(2, 100), (40, 60)])])
def test_wide_rows(B, H, hk, D, seqs):
    """Rows of more than 8192 features through all four calls."""
    s = Setup(B, seqs, H=H, hk=hk, D=D, page=64, seed=21, stale=0.0)
    assert H * D > 8192
    q, k, v = s.new_rows(True)
    rot = B.Rotation(torch.from_numpy(FREQ(D // 2)).cuda())
    s.q = B.cache_append(s.p, s.cache, q, k, v, s.row_offsets, s.dlens, rotation=rot)
    tok = np.concatenate([co.tokens(s.ro, s.lens, b) for b in range(len(seqs))])
    for x, got in ((q, s.q), (k, None)):
        want = co.rotate(f64(x), tok, FREQ(D // 2).astype(np.float64), "halves")
        if got is None:
            seq = np.concatenate([[b] * n for b, (n, _) in enumerate(seqs)]).astype(int)
            pg = torch.from_numpy(s.table[seq, tok // s.page].astype(np.int64)).cuda()
            slot = torch.from_numpy(tok % s.page).cuda()
            got = s.cache.k[pg, :, slot]
            assert torch.equal(s.cache.v[pg, :, slot], v)
        part = np.abs(f64(x)) + np.abs(np.roll(f64(x), D // 2, axis=-1))
        assert (np.abs(f64(got) - want) <= BF * np.abs(want) + (1 + BF) * 8 * U * part).all()
    got = attn(s, B)
    sel = B.cache_select(s.p, s.cache, s.q, s.row_offsets, s.dlens, 3)
    by = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, sel)
    torch.cuda.synchronize()
    s.check(got, s.reference(), False)
    want = co.select(f64(s.q), f64(s.cache.mean), s.table, s.page, s.ro, s.lens, 3, 1, 1)
    assert (sel.cpu().numpy() == want).all()
    s.check(by, s.reference(want), False)


# ---------------------------------------------------------------------------
# Use

def step(s, B, rot, q, k, v, ws, out, stream=None):
    """One step of a program: append, attention, selection, attention over pages."""
    qr, sel, a, b = out
    B.cache_append(s.p, s.cache, q, k, v, s.row_offsets, s.dlens, rotation=rot, out=qr,
                   stream=stream)
    B.cache_attn(s.p, s.cache, qr, s.row_offsets, s.dlens, out=a, workspace=ws, stream=stream)
    B.cache_select(s.p, s.cache, qr, s.row_offsets, s.dlens, sel.shape[2], out=sel, workspace=ws,
                   stream=stream)
    B.cache_attn_pages(s.p, s.cache, qr, s.row_offsets, s.dlens, sel, out=b, workspace=ws,
                       stream=stream)


def outputs(s, n_sel):
    e = lambda *shape, dt=torch.bfloat16: torch.zeros(*shape, dtype=dt, device="cuda")
    M = s.p.total_kept
    pair = lambda: (e(M, s.H, s.D), e(M, s.H, dt=torch.float32))
    return e(M, s.H, s.D), e(M, s.hk, n_sel, dt=torch.int32), pair(), pair()


def flat(out):
    return [out[0], out[1], *out[2], *out[3]]


def test_a_step_captured_and_replayed(B):
    """A captured step, replayed while its lengths, rows and tables change under it,
    with eager work between; every replay against the eager step."""
    s = Setup(B, [(2, 1100), (1, 30), (1, 700)], H=8, hk=2, D=128, page=64, extra_rows=2, seed=7)
    s.p.L_max = 1200
    s.table = np.concatenate([s.table, np.full((3, 3), -1, np.int32)], 1)
    s.cache.page_table = dev(s.table)
    rot = B.Rotation(torch.from_numpy(FREQ(64)).cuda())
    q, k, v = s.new_rows(True)
    ws = torch.empty(max(B.workspace_bytes_cache(s.p, s.cache),
                         B.workspace_bytes_cache(s.p, s.cache, 9)), dtype=torch.uint8, device="cuda")
    out, ref = outputs(s, 9), outputs(s, 9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(s, B, rot, q, k, v, ws, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s, B, rot, q, k, v, ws, out)
    for turn, (ro, lens) in enumerate([([0, 2, 3, 4], [1100, 30, 700]), ([0, 1, 1, 3], [3, 30, 650]),
                                       ([0, 2, 4, 6], [1088, 31, 64]), ([0, 0, 0, 0], [0, 0, 0])]):
        s.row_offsets.copy_(dev(ro))
        s.dlens.copy_(dev(lens))
        q.normal_()
        k.normal_()
        before = [x.clone() for x in (s.cache.k, s.cache.v, s.cache.mean)]
        for o in flat(out) + flat(ref):
            o.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        after = [x.clone() for x in (s.cache.k, s.cache.v, s.cache.mean)]
        for x, y in zip((s.cache.k, s.cache.v, s.cache.mean), before):
            x.copy_(y)
        step(s, B, rot, q, k, v, None, ref)
        torch.cuda.synchronize()
        for x, y in zip(flat(out), flat(ref)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), turn
        for x, y in zip((s.cache.k, s.cache.v, s.cache.mean), after):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), turn
        M = ro[-1]
        assert all((o[M:] == 5).all() for o in flat(out))


@pytest.mark.parametrize("tall", [False, True])
def test_prefixes_and_runs_captured_and_replayed(B, tall):
    """Shared prefixes, and many new tokens in runs: a captured call replayed while rows,
    lengths and prefixes change under it, with eager work between; its own workspace."""
    n = 40 if tall else 2
    s = Setup(B, [(n, 2500), (n, 2300), (n, 2200), (n, 2400)], H=16, hk=8, D=128, page=64, seed=22,
              shared=[(0, i, 2100) for i in (1, 2, 3)])
    s.table = np.concatenate([s.table, np.full((4, 40), -1, np.int32)], 1)
    s.cache.page_table = dev(s.table)
    s.p.L_max = 4300                                  # (64 MB and more: prefixes are items)
    assert 4 * 4 * 8 * s.p.L_max * 128 >= 64 << 20
    ids, P = dev([0] * 4), dev([2100] * 4)
    call = lambda out: attn(s, B, prefix_ids=ids, prefix_lens=P, out=out)
    new = lambda: (torch.empty_like(s.q), torch.empty(s.p.total_kept, s.H, device="cuda"))
    out, ref = new(), new()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for ro, lens, i, pl in (([0, n, 2 * n, 3 * n, 4 * n], [2500, 2300, 2200, 2400], 0, 2100),
                            ([0, 0, n, n, 2 * n], [9, 2250, 0, 2150], 3, 2048),
                            ([0, 1, 2, 3, 4], [2100, 2120, 2200, 700], 0, 2100),
                            ([0] * 5, [0] * 4, 0, 2100),
                            ([0, n, n + 1, n + 2, 2 * n], [2400, 2200, 33, 2300], -1, 2100)):
        for x, y in ((s.row_offsets, ro), (s.dlens, lens), (ids, [i] * 4), (P, [pl] * 4)):
            x.copy_(dev(y))
        s.q.normal_()
        for x in (*out, *ref):
            x.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        call(ref)
        torch.cuda.synchronize()
        for x, y in zip(out, ref):
            assert torch.equal(x, y), (ro, lens)
        s.ro, s.lens = np.array(ro, np.int32), np.array(lens, np.int32)
        s.check(out, s.reference(), False)
        assert (out[0][ro[-1]:] == 5).all()


def test_two_streams_at_once(B):
    """Two sequences' steps on streams of their own, workspaces and outputs made by the
    calls."""
    setups = [Setup(B, [(1, 3000)], seed=8), Setup(B, [(3, 2500), (1, 10)], H=16, hk=2, seed=9)]
    want = [attn(s, B) for s in setups]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in setups]
    got = []
    for turn in range(6):
        got.append([B.cache_attn(s.p, s.cache, s.q, s.row_offsets, s.dlens, stream=st)
                    for s, st in zip(setups, streams)])
    torch.cuda.synchronize()
    for turn in got:
        for a, b in zip(turn, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_memory_of_a_call_on_another_stream(B):
    """Workspaces and outputs that calls on two streams make in turn: never a block that
    the other stream may still use, and the same results."""
    s = Setup(B, [(1, 3000), (2, 1500)], H=16, hk=2, seed=18)
    want = attn(s, B)
    sel = B.cache_select(s.p, s.cache, s.q, s.row_offsets, s.dlens, 40)
    by = B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens, sel)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    n = 1 << 20
    here = B._fresh_workspace(n, "cuda").data_ptr()          # (released: the current stream's)
    other = B._fresh_workspace(n, "cuda", side).data_ptr()
    assert other != here and B._fresh_workspace(n, "cuda").data_ptr() == here
    got = []
    for turn in range(8):
        for stream in (None, side):
            args = (s.p, s.cache, s.q, s.row_offsets, s.dlens)
            got.append((B.cache_attn(*args, stream=stream),
                        B.cache_attn_pages(*args, sel, stream=stream),
                        B.cache_select(*args, 40, stream=stream)))
        if turn % 2:
            got = got[-3:]                                   # (the others' memory is free again)
    torch.cuda.synchronize()
    for a, b, c in got:
        for x, y in zip((*a, *b, c), (*want, *by, sel)):
            assert torch.equal(x, y)


def test_from_the_route_to_an_answer(B):
    """The calls in the order of a program: kept tokens routed to their passages, the
    layer that makes their queries, keys and values, a cache that takes them in, and
    tokens appended one by one, over all tokens and over selected pages."""
    from paper_2607_25422_amd import workloads as wls
    batch = wls.make_batch("llava_bf16", 2026, B=3)
    db = B.to_device(batch)
    H, D, hk = db.p.H, db.p.d_h, 4
    kept, fused, _ = B.route_fused(db)
    g = torch.Generator(device="cuda").manual_seed(2)
    wide = (H + 2 * hk) * D
    W = (torch.randn(wide, db.p.d, generator=g, device="cuda") / 32).bfloat16()
    packed = B.pack_dense(db.p, W)
    x = B.gather_dense(db.p, fused.reshape(-1, db.p.d), packed, wide)
    ko = db.kept_offsets.cpu().numpy()
    lens = np.diff(ko).astype(np.int32)
    need = -(-(lens + 40) // 32)
    table = np.full((3, int(need.max())), -1, np.int32)
    ids = np.random.default_rng(3).permutation(int(need.sum())).astype(np.int32)
    for b, e in enumerate(np.cumsum(need)):
        table[b, :need[b]] = ids[e - need[b]:e]
    cache = B.new_kv_cache(int(need.sum()), hk, 32, D, dev(table))
    rot = B.Rotation(torch.from_numpy(FREQ(D // 2)).cuda())

    def split(y):
        return [c.unflatten(1, (-1, D)) for c in (y[:, :H * D], y[:, H * D:(H + hk) * D],
                                                  y[:, (H + hk) * D:])]
    p = B.make_problem("bf16", B=3, d=db.p.d, H=H, d_h=D, kept_offsets=ko)
    p.L_max = int(lens.max())
    # kept tokens rotate by their place in the image
    q = B.cache_append(p, cache, *split(x), db.kept_offsets, dev(lens), rotation=rot,
                       positions=kept)
    O, lse = B.cache_attn(p, cache, q, db.kept_offsets, dev(lens))
    s = Setup.__new__(Setup)
    s.D, s.scale, s.q, s.cache, s.ro, s.lens, s.table = D, float(p.sm_scale), q, cache, ko, lens, table
    s.check((O, lse), s.reference(), False)
    ro = np.arange(4, dtype=np.int32)
    for t in range(35):
        lens = lens + 1
        y = torch.randn(3, wide, generator=g, device="cuda").bfloat16()
        p1 = B.make_problem("bf16", B=3, d=db.p.d, H=H, d_h=D, kept_offsets=ro)
        p1.L_max = int(lens.max())
        q = B.cache_append(p1, cache, *split(y), dev(ro), dev(lens), rotation=rot)
        sel = B.cache_select(p1, cache, q, dev(ro), dev(lens), 3)
        got = B.cache_attn(p1, cache, q, dev(ro), dev(lens))
        by = B.cache_attn_pages(p1, cache, q, dev(ro), dev(lens), sel)
    s.q, s.ro, s.lens = q, ro, lens
    s.check(got, s.reference(), False)
    want = co.select(f64(q), f64(cache.mean), table, 32, ro, lens, 3, 1, 1)
    assert (sel.cpu().numpy() == want).all()
    s.check(by, s.reference(want), False)


def test_refused_tensors(B):
    s = Setup(B, [(1, 40)])
    q, k, v = s.new_rows(False)
    app = lambda *a, **kw: B.cache_append(s.p, s.cache, *a, s.row_offsets, s.dlens, **kw)
    for bad in ((q.float(), k, v), (q, k[:, :1], v), (q, k, v.transpose(1, 2)), (q.cpu(), k, v)):
        with pytest.raises(ValueError):
            app(*bad)
    with pytest.raises(ValueError):
        attn(s, B, prefix_ids=dev([0]).float(), prefix_lens=dev([0]))
    with pytest.raises(B.SkipError):
        attn(s, B, prefix_ids=dev([0]))
    with pytest.raises(ValueError):
        B.cache_attn_pages(s.p, s.cache, s.q, s.row_offsets, s.dlens,
                           torch.zeros(1, 1, 3, dtype=torch.int32, device="cuda"))
