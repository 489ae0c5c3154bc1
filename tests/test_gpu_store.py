"""Passages held in 4 bits: the store written and read back against the oracle
bit by bit, and the bipartite attention over it against a float64 softmax over the
held values."""
import math
import sys

import numpy as np
import pytest
import torch

import oracle as orc

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def B():
    from paper_2607_25422_amd import binding
    return binding


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int32)


class Held:
    """Passages on the device, in a store, and as held (float64, on the host)."""

    def __init__(self, B, Ls, H, Hkv, D, seed, dtype="bf16", make=None, first=0):
        g = torch.Generator().manual_seed(seed)
        n = sum(Ls)
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        K, V = (torch.randn(n, Hkv, D, generator=g) for _ in range(2))
        if make:
            K, V = make(K), make(V)
        self.K, self.V = K.to(self.dt), V.to(self.dt)
        self.Ls, self.H, self.Hkv, self.D = Ls, H, Hkv, D
        self.off = cum(Ls)
        self.blocks, end = B.passage_blocks(self.off, first)
        self.p = B.make_problem(dtype, B=1, d=H * D, H=H, d_h=D, passage_offsets=self.off,
                                query_passages=[0, len(Ls)])
        self.store = B.new_kv_store(Hkv, D, end + 2)
        self.po, self.pb = dev(self.off), dev(self.blocks)

    def write(self, B, want_keys=False):
        return B.quantize_passages(self.p, self.store, self.K.cuda(), self.V.cuda(), self.po,
                                   self.pb, want_keys)

    def held1(self):
        """As held, of the passages that were written."""
        return self.held(cum(self.Ls))

    def held(self, off=None):
        Ko, Vo = [], []
        off = self.off if off is None else off
        for a, b in zip(off[:-1], off[1:]):
            k, v = orc.held_passage(self.K[a:b].double().numpy(), self.V[a:b].double().numpy())
            Ko.append(k)
            Vo.append(v)
        return np.concatenate(Ko), np.concatenate(Vo)


def spread(x):
    """Blocks of very different sizes, zeros, ties and sevens among them."""
    n = x.shape[0]
    x = x * torch.exp2(torch.arange(n).remainder(41).sub(20).float())[:, None, None]
    x = (x * 8).round() / 8                       # many ties at the larger sizes
    x[::5] = 0.0
    x[1::7, :, ::3] = 7.0
    x[2::7, :, 1::3] = -7.03125
    x[3::11] *= -0.0
    return x


# blocks of very small and very large numbers
def tiny(x):
    return x * 2.0 ** -126


def huge(x):
    return x * 2.0 ** 124


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,Hkv", [(64, 4, 4), (64, 6, 3), (128, 5, 5), (128, 8, 1)])
@pytest.mark.parametrize("make", [None, spread, tiny, huge])
def test_store_round_trip(B, D, H, Hkv, dtype, make):
    Ls = [1, 31, 32, 33, 70]
    say(f"store {dtype} D={D} Hkv={Hkv} make={make.__name__ if make else None}")
    x = Held(B, Ls, H, Hkv, D, 5, dtype, make, first=1)
    x.store.data.fill_(0xA5)
    x.write(B)
    K, V = B.dequantize_passages(x.p, x.store, x.po, x.pb)
    torch.cuda.synchronize()
    Ko, Vo = x.held()
    assert np.array_equal(K.cpu().double().numpy(), Ko)
    assert np.array_equal(V.cpu().double().numpy(), Vo)
    # the record before the first and those after the last are as they were
    rec = x.store.data.view(x.store.n_blocks, -1).cpu()
    assert (rec[0] == 0xA5).all() and (rec[-2:] == 0xA5).all()


@pytest.mark.parametrize("D", [64, 128])
def test_record_layout(B, D):
    """The bytes of a record as the header lays them out."""
    L, Hkv = 45, 2
    x = Held(B, [L], 2, Hkv, D, 6)
    x.write(B)
    torch.cuda.synchronize()
    rec = x.store.data.cpu().numpy().reshape(-1, Hkv, 34 * D)
    K = np.zeros((64, Hkv, D))
    V = np.zeros((64, Hkv, D))
    K[:L], V[:L] = x.K.double().numpy(), x.V.double().numpy()
    for blk in range(2):
        for h in range(Hkv):
            want = np.zeros(34 * D, dtype=np.uint8)
            for t in range(32):
                for c in range(D // 32):
                    codes, s, _ = orc.held_block(K[32 * blk + t, h, 32 * c:32 * c + 32])
                    at = ((t // 16 * (D // 32) + c) * 16 + t % 16) * 16
                    want[at:at + 16] = [codes[2 * i] | codes[2 * i + 1] << 4 for i in range(16)]
                    want[32 * D + (c % 2 * 16 + t % 16) * (D // 32) + t // 16 * (D // 64) +
                         c // 2] = s
            for f in range(D):
                codes, s, _ = orc.held_block(V[32 * blk:32 * blk + 32, h, f])
                at = 16 * D + 16 * f
                want[at:at + 16] = [codes[2 * i] | codes[2 * i + 1] << 4 for i in range(16)]
                want[33 * D + f % 32 * (D // 32) + f // 32] = s
            assert np.array_equal(rec[blk, h], want), (blk, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 64), (24, 3, 128), (32, 32, 128)])
def test_mean_keys(B, H, Hkv, D, dtype):
    """The float rounding of the float64 mean (its sum's own rounding, at most L
    2^-53, can move a float at a border only)."""
    Ls = [1, 4, 17, 133]
    say(f"mean keys {dtype} H={H} Hkv={Hkv} D={D}")
    x = Held(B, Ls, H, Hkv, D, 7, dtype)
    keys = x.write(B, want_keys=True)
    torch.cuda.synchronize()
    for j, (a, b) in enumerate(zip(x.off[:-1], x.off[1:])):
        k = x.K[a:b].double()
        want = k.mean(0).repeat_interleave(H // Hkv, 0).reshape(-1)
        bound = (2.0 ** -24 * want.abs() + 2.0 ** -50 * k.abs().mean(0).max()).numpy()
        got = keys[j].cpu().double()
        assert (np.abs((got - want).numpy()) <= bound).all()


# ---------------------------------------------------------------------------
# Attention

def rows_of(M, H, D, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(M, H, D, generator=g).bfloat16()


def random_graph(ks, Ps, seed):
    """Neighbours of every row: none for some, every passage for some."""
    rng = np.random.default_rng(seed)
    out = []
    for k, P in zip(ks, Ps):
        for i in range(k):
            n = min(P, int(rng.choice([0, 1, 2, 4, P])))
            out.append(sorted(rng.choice(P, n, replace=False).tolist()))
    return out


def reference(Q, K, V, nb, ks, Ps, off, scale, G, o_f32=False, piece=None):
    """O, LSE in float64 and a bound of the kernel's error before the output's own
    rounding: the logits' products are exact and summed in float32 (at most D
    roundings of 2^-24 of the sum of magnitudes, the scale's and the exponent's
    rounding a few more of the logit), a weight enters as a half float, half a step
    of 2^-10 off (three bf16 pieces for float output: 2^-24; two where a held value
    is no half float: 2^-16; a weight below 2^-14 is off by at most 2^-25 of the
    largest), the float32 sums of n weights by n 2^-24; twice for numerator and
    denominator."""
    piece = piece or (2.0 ** -24 if o_f32 else 2.0 ** -11)
    O = np.zeros(Q.shape)
    lse = np.full(Q.shape[:2], -np.inf)
    bound = np.zeros(Q.shape[:2])
    lbound = np.zeros(Q.shape[:2])
    r = p = 0
    D = Q.shape[2]
    for k, P in zip(ks, Ps):
        for i in range(r, r + k):
            tok = [t for j in nb[i] for t in range(off[p + j], off[p + j + 1])]
            if not tok:
                continue
            for h in range(Q.shape[1]):
                kk, vv = K[tok, h // G], V[tok, h // G]
                z = scale * (kk @ Q[i, h])
                m = z.max()
                w = np.exp(z - m)
                O[i, h] = w @ vv / w.sum()
                lse[i, h] = m + math.log(w.sum())
                mag = abs(scale) * (np.abs(kk) @ np.abs(Q[i, h])).max()
                dz = 2.0 ** -24 * (D + 8) * mag
                bound[i, h] = 2 * (dz + piece + 2.0 ** -24 * (len(tok) + 16)) * np.abs(vv).max()
                lbound[i, h] = dz + 2.0 ** -24 * (len(tok) + 16 + 2 * abs(lse[i, h]))
        r += k
        p += P
    return O, lse, bound, lbound


def attend(B, x, Q, nb, ks, Ps, scale, o_f32=False, **kw):
    H, D = Q.shape[1:]
    p = B.make_problem("bf16", B=len(ks), d=H * D, H=H, d_h=D, kept_offsets=cum(ks),
                       passage_offsets=x.off, query_passages=cum(Ps), sm_scale=scale,
                       o_f32=o_f32, total_edges=sum(map(len, nb)), N=kw.pop("N", 0))
    col = dev([j for r in nb for j in r] or [0])[:p.total_edges]
    out = kw.pop("out", None)
    O, lse = B.bipartite_xattn_quant(p, x.store, Q.cuda(), dev(cum(ks)), x.po, x.pb, dev(cum(Ps)),
                                     edges=(dev(cum([len(r) for r in nb])), col), out=out, **kw)
    return O, lse


def check(O, lse, ref, o_f32, what):
    Or, Lr, bound, lbound = ref
    O, lse = O.cpu().double().numpy(), lse.cpu().double().numpy()
    out = np.abs(Or) * (2.0 ** -24 if o_f32 else 2.0 ** -8)
    over = np.abs(O - Or) - out - bound[..., None]
    assert not np.isnan(O).any()
    empty = np.isinf(Lr)
    assert (lse[empty] == -np.inf).all() and (O[empty] == 0).all()
    dl = np.abs(np.where(empty, 0, lse) - np.where(empty, 0, Lr)) - lbound
    say(f"{what}: largest excess over the bound O {over.max():.2e} LSE {dl.max():.2e}, "
        f"error {np.abs(O - Or).max():.2e}")
    assert over.max() <= 0 and dl.max() <= 0


@pytest.mark.parametrize("D,H,Hkv", [(64, 2, 2), (64, 6, 2), (64, 8, 1), (128, 2, 2), (128, 10, 2)])
@pytest.mark.parametrize("ks,Ps,Ls", [
    ([1], [1], [1]),
    ([1], [3], [33, 1, 64]),
    ([2, 0, 35], [2, 1, 4], [65, 127, 5, 31, 96, 32, 200]),
    ([33, 7], [0, 5], [1, 63, 64, 129, 40]),
    ([5], [20], [3] * 19 + [70]),
])
@pytest.mark.parametrize("o_f32", [False, True])
def test_attention_shapes(B, D, H, Hkv, ks, Ps, Ls, o_f32):
    say(f"store attention D={D} H={H}/{Hkv} ks={ks} Ps={Ps} Ls={Ls}")
    x = Held(B, Ls, H, Hkv, D, 8)
    x.write(B)
    Q = rows_of(sum(ks), H, D, 9)
    nb = random_graph(ks, Ps, 10)
    scale = 1.5 / math.sqrt(D)
    O, lse = attend(B, x, Q, nb, ks, Ps, scale, o_f32)
    torch.cuda.synchronize()
    ref = reference(Q.double().numpy(), *x.held(), nb, ks, Ps, x.off, scale, H // Hkv, o_f32)
    check(O, lse, ref, o_f32, "shapes")


def wide_values(x):
    """Features from 2^-40 to 2^40: no half floats."""
    return x * torch.exp2(torch.arange(x.shape[-1]).remainder(9).sub(4).float() * 10)


def one_wide(x):
    """Half floats but for one feature of the later tokens."""
    x = x.clone()
    x[100:, -1, 5] *= 2.0 ** 30
    return x


@pytest.mark.parametrize("make", [wide_values, one_wide])
@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_values_that_are_no_half_floats(B, D, nq, make):
    """Both forms (few rows; from 768 tiles of 32 rows on), elementwise against each
    feature's own size."""
    H, ks, Ps = 4, [9] * nq, [3] * nq
    x = Held(B, [90, 64, 33], H, H, D, 25)
    x.V = make(x.V.float()).to(x.dt)
    x.write(B)
    x.off, x.po = cum([90, 64, 33] * nq), dev(cum([90, 64, 33] * nq))
    x.pb = dev(np.tile(x.blocks, nq))
    say(f"store attention wide values D={D} nq={nq} {make.__name__}")
    Q = rows_of(9, H, D, 26)
    nb = random_graph([9], [3], 27)
    O, lse = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, ks, Ps, 0.2)
    torch.cuda.synchronize()
    K, V = x.held1()
    ref = reference(Q.double().numpy(), K, V, nb, [9], [3], cum([90, 64, 33]), 0.2, 1)
    size = np.abs(V).max(0)[None]                     # of each head's feature
    lim = ref[2] / np.maximum(np.abs(V).max(), 1e-300)
    O = O.cpu().double().numpy().reshape(nq, 9, H, D)
    assert (O == O[:1]).all()
    err = np.abs(O[0] - ref[0])
    assert (err <= np.abs(ref[0]) * 2.0 ** -8 + lim.max() * size).all()


@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_attention_scales(B, scale):
    ks, Ps, Ls = [40], [3], [70, 20, 64]
    x = Held(B, Ls, 2, 2, 64, 11)
    x.write(B)
    Q = rows_of(40, 2, 64, 12)
    nb = random_graph(ks, Ps, 13)
    O, lse = attend(B, x, Q, nb, ks, Ps, scale)
    torch.cuda.synchronize()
    check(O, lse, reference(Q.double().numpy(), *x.held(), nb, ks, Ps, x.off, scale, 1), False,
          f"scale {scale}")


@pytest.mark.parametrize("k,H,Hkv,nq", [(200, 4, 2, 2), (97, 32, 4, 1), (64, 3, 3, 9)])
def test_attention_row_chunks(B, k, H, Hkv, nq):
    """Rows of a question over several items, some rows compared."""
    D, P = 64, 3
    Ls = [40, 65, 10] * nq
    ks, Ps = [k] * nq, [P] * nq
    say(f"store attention chunks k={k} H={H}/{Hkv} nq={nq}")
    x = Held(B, Ls, H, Hkv, D, 14)
    x.write(B)
    Q = rows_of(k * nq, H, D, 15)
    nb = random_graph(ks, Ps, 16)
    O, lse = attend(B, x, Q, nb, ks, Ps, 0.2, True)
    torch.cuda.synchronize()
    ref = reference(Q.double().numpy(), *x.held(), nb, ks, Ps, x.off, 0.2, H // Hkv, True)
    check(O, lse, ref, True, "chunks")


@pytest.mark.parametrize("D", [64, 128])
def test_attention_long_passages_split(B, D):
    """Few rows over many tokens: items split over workgroups, joined again."""
    ks, Ps, Ls = [1, 2], [4, 3], [900, 1, 1500, 333, 64, 700, 2000]
    say(f"store attention split D={D}")
    x = Held(B, Ls, 4, 1, D, 17)
    x.write(B)
    Q = rows_of(3, 4, D, 18)
    nb = [[0, 1, 2, 3], [0, 2], []]
    O, lse = attend(B, x, Q, nb, ks, Ps, 0.3, True)
    torch.cuda.synchronize()
    ref = reference(Q.double().numpy(), *x.held(), nb, ks, Ps, x.off, 0.3, 4, True)
    check(O, lse, ref, True, "split")


def test_attention_graph_from_keys(B):
    """The graph built from the mean keys, rows in place through the kept indices;
    equal to the call on the same graph given, and to the oracle's edges."""
    H, Hkv, D, N, ks, Ps = 4, 2, 64, 90, [37, 12], [5, 3]
    Ls = [33, 40, 7, 64, 90, 12, 50, 31]
    x = Held(B, Ls, H, Hkv, D, 19)
    keys = x.write(B, want_keys=True)
    g = torch.Generator().manual_seed(20)
    V = torch.randn(2, N, H * D, generator=g).bfloat16()
    idx = torch.cat([torch.randperm(N, generator=g)[:k].sort().values for k in ks]).int()
    rows = torch.cat([V[0, idx[:37].long()], V[1, idx[37:].long()]])
    p = B.make_problem("bf16", B=2, N=N, d=H * D, H=H, d_h=D, kept_offsets=cum(ks),
                       passage_offsets=x.off, query_passages=cum(Ps), sm_scale=0.1,
                       avg_degree=2.0)
    rp = torch.empty(sum(ks) + 1, dtype=torch.int32, device="cuda")
    col = torch.empty(sum(ks) * 5, dtype=torch.int32, device="cuda")
    O = torch.empty(sum(ks), H, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(sum(ks), H, device="cuda")
    B.skip_bipartite_xattn_quant(p, x.store, V.cuda(), dev(cum(ks)), x.po, x.pb, dev(cum(Ps)), O,
                                 lse, kept_idx=idx.cuda(), passage_keys=keys,
                                 edge_rowptr_out=rp, edge_col_out=col)
    torch.cuda.synchronize()
    adj = [orc.bsca_edges(orc.cosine_matrix(rows[a:b].double().numpy(),
                                            keys[c:d].cpu().double().numpy()), 2.0)
           for a, b, c, d in ((0, 37, 0, 5), (37, 49, 5, 8))]
    nb = [np.nonzero(r)[0].tolist() for a in adj for r in a]
    assert rp.cpu().tolist() == cum([len(r) for r in nb]).tolist()
    assert col.cpu().tolist()[:sum(map(len, nb))] == [j for r in nb for j in r]
    O2, lse2 = attend(B, x, rows.view(-1, H, D), nb, ks, Ps, 0.1)
    torch.cuda.synchronize()
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    check(O, lse, reference(rows.view(-1, H, D).double().numpy(), *x.held(), nb, ks, Ps, x.off,
                            0.1, 2), False, "from keys")


def test_attention_shared_passages_and_far_records(B):
    """Two questions that name one stored passage, and records past 4 GiB: the
    same bits as from a small store."""
    H, D, L = 8, 128, 100
    per = 34 * D * H
    n_blocks = (1 << 32) // per + 40
    x = Held(B, [L], H, H, D, 21)
    x.write(B)
    far = B.KvStore(torch.empty(n_blocks * per, dtype=torch.uint8, device="cuda"), H, n_blocks)
    at = n_blocks - 7
    B.quantize_passages(x.p, far, x.K.cuda(), x.V.cuda(), x.po, dev([at]))
    off = cum([L, L])
    p = B.make_problem("bf16", B=2, d=H * D, H=H, d_h=D, kept_offsets=[0, 3, 8],
                       passage_offsets=off, query_passages=[0, 1, 2], total_edges=8,
                       sm_scale=0.1)
    Q = rows_of(8, H, D, 22).cuda()
    graph = dev(np.arange(9)), dev(np.zeros(8))
    args = dev([0, 3, 8]), dev(off)
    a = B.bipartite_xattn_quant(p, x.store, Q, *args, dev([0, 0]), dev([0, 1, 2]), edges=graph)
    b = B.bipartite_xattn_quant(p, far, Q, *args, dev([at, at]), dev([0, 1, 2]), edges=graph)
    K, V = B.dequantize_passages(x.p, far, x.po, dev([at]))
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert np.array_equal(K.cpu().double().numpy(), x.held()[0])
    assert torch.isfinite(a[1]).all()


def test_attention_gate_mask_and_other_stream(B):
    """A dropped passage gets no edge; the call on a stream that is not current."""
    H, D, ks, Ps = 2, 64, [20], [4]
    x = Held(B, [33, 40, 7, 64], H, H, D, 23)
    keys = x.write(B, want_keys=True)
    Q = rows_of(20, H, D, 24).cuda()
    keep = torch.tensor([1, 0, 1, 1], dtype=torch.uint8, device="cuda")
    p = B.make_problem("bf16", B=1, d=H * D, H=H, d_h=D, kept_offsets=cum(ks),
                       passage_offsets=x.off, query_passages=cum(Ps), avg_degree=2.0)
    O = torch.full((20, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((20, H), float("nan"), device="cuda")
    rp = torch.empty(21, dtype=torch.int32, device="cuda")
    col = torch.full((80,), -1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    B.skip_bipartite_xattn_quant(p, x.store, Q, dev(cum(ks)), x.po, x.pb, dev(cum(Ps)), O, lse,
                                 passage_keys=keys, passage_keep=keep, edge_rowptr_out=rp,
                                 edge_col_out=col, stream=s)
    s.synchronize()
    n = int(rp[-1])
    assert n == 40 and 1 not in col[:n].tolist()
    cols, ptr = col.tolist(), rp.tolist()
    nb = [cols[ptr[i]:ptr[i + 1]] for i in range(20)]
    check(O, lse, reference(Q.cpu().double().numpy(), *x.held(), nb, ks, Ps, x.off,
                            1 / math.sqrt(D), 1), False, "gate mask")
