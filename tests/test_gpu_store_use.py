"""The calls around the 4-bit store as they are used together: a question's whole
way, captured graphs, two calls at once; and what no single call's test reaches:
batches taken out of order, graphs with columns that do not exist, records outside
the store, infinities behind a mask."""
import math

import numpy as np
import pytest
import torch

import oracle as orc
from paper_2607_25422_amd import workloads as wls
from test_gpu_capture import check_replays
from test_gpu_dense import act64
from test_gpu_store import (Held, attend, check, cum, dev, random_graph, reference, rows_of, say)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_25422_amd import binding
    return binding


# ---------------------------------------------------------------------------
# Batches

def some_of(x, O, lse, Q, nb, ks, Ps, scale, G, o_f32, questions, heads):
    """The reference of some questions and key heads."""
    ko, po, qo = cum(ks), x.off, cum(Ps)
    for b in questions:
        r, t = slice(ko[b], ko[b + 1]), slice(po[qo[b]], po[qo[b + 1]])
        off = po[qo[b]:qo[b + 1] + 1] - po[qo[b]]
        for hk in heads:
            h = slice(hk * G, hk * G + G)
            K, V = (np.concatenate([np.zeros((0, 1, x.D))] + [
                orc.held_passage(x.K[t][a:c, hk:hk + 1].double().numpy(),
                                 x.V[t][a:c, hk:hk + 1].double().numpy())[i]
                for a, c in zip(off[:-1], off[1:])]) for i in (0, 1))
            if ks[b]:
                ref = reference(Q[r, h].double().numpy(), K, V, nb[r], [ks[b]], [Ps[b]], off, scale,
                                G, o_f32)
                check(O[r, h], lse[r, h], ref, o_f32, f"question {b} key head {hk}")


@pytest.mark.parametrize("o_f32", [False, True])
@pytest.mark.parametrize("index", [False, True])
@pytest.mark.parametrize("nq,top,D,H,Hkv", [(50, 250, 64, 32, 16), (60, 130, 128, 16, 16),
                                            (90, 40, 64, 36, 12), (30, 100, 128, 32, 32)])
def test_ragged_batches_of_many_items(B, nq, top, D, H, Hkv, o_f32, index):
    """The form of many rows: questions of mixed sizes (taken longest first up to
    64 of them), some without rows or passages, one of 64 passages, some of few."""
    rng = np.random.default_rng(31)
    G = H // Hkv
    ks = [int(k) for k in rng.choice([0, 1, 3, 9, 20], nq)]
    Ps = [int(p) for p in rng.choice([0, 1, 2, 3], nq)]
    ks[nq // 2], Ps[nq // 2] = top, 2
    ks[3], Ps[3] = 33, 64
    assert nq * Hkv * math.ceil(sum(ks) * G / nq / 32) >= 768      # else the form of few rows
    Ls = [int(v) for v in rng.choice([1, 5, 31, 32, 33, 64, 65, 130], sum(Ps))]
    say(f"ragged batch nq={nq} D={D} H={H}/{Hkv} f32={o_f32} index={index}")
    x = Held(B, Ls, H, Hkv, D, 32)
    x.write(B)
    nb = random_graph(ks, Ps, 33)
    if index:
        N = top + 7
        V = rows_of(nq * N, H, D, 34)
        g = torch.Generator().manual_seed(35)
        idx = [torch.randperm(N, generator=g)[:k].sort().values for k in ks]
        Q = torch.cat([V.view(nq, N, H, D)[b, i] for b, i in enumerate(idx)])
        O = torch.empty(sum(ks), H, D, device="cuda",
                        dtype=torch.float32 if o_f32 else torch.bfloat16)
        lse = torch.empty(sum(ks), H, device="cuda")
        p = B.make_problem("bf16", B=nq, N=N, d=H * D, H=H, d_h=D, kept_offsets=cum(ks),
                           passage_offsets=x.off, query_passages=cum(Ps), sm_scale=0.2,
                           o_f32=o_f32, total_edges=sum(map(len, nb)))
        B.skip_bipartite_xattn_quant(
            p, x.store, V.cuda(), dev(cum(ks)), x.po, x.pb, dev(cum(Ps)), O, lse,
            kept_idx=torch.cat(idx).int().cuda(), edge_rowptr=dev(cum([len(r) for r in nb])),
            edge_col=dev([j for r in nb for j in r]))
    else:
        Q = rows_of(sum(ks), H, D, 34)
        O, lse = attend(B, x, Q, nb, ks, Ps, 0.2, o_f32)
    torch.cuda.synchronize()
    rowless = torch.tensor([not r for r in nb])
    O, lse = O.cpu(), lse.cpu()
    assert not O[rowless].any() and (lse[rowless] == -math.inf).all()
    assert torch.isfinite(O).all() and torch.isfinite(lse[~rowless]).all()
    some_of(x, O, lse, Q, nb, ks, Ps, 0.2, G, o_f32,
            [3, nq // 2, 0, nq - 1] + rng.choice(nq, 4).tolist(), [0, Hkv - 1])


@pytest.mark.parametrize("ks,Ps", [([0, 0], [2, 1]), ([3, 2], [0, 0]), ([0], [0])])
def test_nothing_to_attend(B, ks, Ps):
    """No rows, or no passages: nothing, or zeros and -inf."""
    x = Held(B, [40] * sum(Ps), 2, 2, 64, 36)
    x.write(B)
    Q = rows_of(sum(ks), 2, 64, 37)
    O, lse = attend(B, x, Q, [[] for _ in range(sum(ks))], ks, Ps, 0.2)
    torch.cuda.synchronize()
    assert O.shape[0] == sum(ks) and not O.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("nq", [1, 200])
def test_columns_twice_and_outside(B, nq):
    """A neighbour named twice counts once, columns that are no passage not at all."""
    H, k, P, Ls = 4, 5, 3, [40, 33, 64]
    x = Held(B, Ls, H, H, 64, 38)
    x.write(B)
    x.off, x.po, x.pb = cum(Ls * nq), dev(cum(Ls * nq)), dev(np.tile(x.blocks, nq))
    Q = rows_of(k, H, 64, 39).repeat(nq, 1, 1)
    plain = [[0, 2], [1], [], [0, 1, 2], [2]]
    wild = [[2, 0, 0, 2, 63, 64], [-1, 1, 1 << 30, -(1 << 31)], [3, -7], [2, 1, 0, 1, 2, 1, 0, 2, 1],
            [2] * 17]
    a = attend(B, x, Q, plain * nq, [k] * nq, [P] * nq, 0.2)
    b = attend(B, x, Q, wild * nq, [k] * nq, [P] * nq, 0.2)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.isfinite(a[0]).all()


# ---------------------------------------------------------------------------
# The store's edges

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_values_are_held_finite(B, dtype):
    def make(v):
        v = v.clone()
        v[3, 0, :3] = torch.tensor([math.inf, -math.inf, 3.3e38])
        v[4] = -3.39e38
        return v
    x = Held(B, [45], 2, 2, 64, 40, dtype, make)
    x.write(B)
    K, V = B.dequantize_passages(x.p, x.store, x.po, x.pb)
    torch.cuda.synchronize()
    Ko, Vo = x.held()
    assert np.isfinite(Ko).all() and np.isfinite(Vo).all()
    assert np.array_equal(K.cpu().double().numpy(), Ko)
    assert np.array_equal(V.cpu().double().numpy(), Vo)


def test_records_outside_the_store(B):
    """Neither written nor read; what is inside is right."""
    H, D, Ls = 2, 64, [70, 40, 33, 64]
    x = Held(B, Ls, H, H, D, 41, first=1)
    x.write(B)
    before = x.store.data.clone()
    n = x.store.n_blocks
    bad = dev([-1, n - 1, 1 << 30, int(x.blocks[3])])     # in part, wholly, wholly outside
    x.store.data.fill_(0x11)
    B.quantize_passages(x.p, x.store, x.K.cuda(), x.V.cuda(), x.po, bad)
    torch.cuda.synchronize()
    rec, old = x.store.data.view(n, -1), before.view(n, -1)
    at = int(x.blocks[3])
    assert torch.equal(rec[at:at + 2], old[at:at + 2])
    # the parts inside: tokens 32 .. of the first passage, 0 .. 31 of the second
    assert torch.equal(rec[0:2], old[int(x.blocks[0]) + 1:int(x.blocks[0]) + 3])
    assert torch.equal(rec[n - 1], old[int(x.blocks[1])])
    others = [i for i in range(2, n - 1) if not at <= i < at + 2]
    assert (rec[others] == 0x11).all()
    out = tuple(torch.full((sum(Ls), H, D), 5.0, dtype=torch.bfloat16, device="cuda")
                for _ in range(2))
    B.dequantize_passages(x.p, x.store, x.po, bad, out)
    Q = rows_of(8, H, D, 42)
    x.pb = bad
    nb = [[3], [0, 1, 2, 3]] * 4
    O, _ = attend(B, x, Q, nb, [8], [4], 0.2)
    torch.cuda.synchronize()
    assert (out[0][:32] == 5.0).all() and (out[1][110:143] == 5.0).all()
    Ko, Vo = x.held()
    assert np.array_equal(out[0][143:].cpu().double().numpy(), Ko[143:])
    ref = reference(Q.double().numpy(), Ko, Vo, nb, [8], [4], x.off, 0.2, 1)
    err = np.abs(O.cpu().double().numpy() - ref[0])[::2]
    assert (err <= 2.0 ** -8 * np.abs(ref[0][::2]) + ref[2][::2, :, None]).all()


@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("o_f32", [False, True])
def test_infinities_behind_the_mask(B, nq, D, o_f32):
    """Passages that a row has no edge to hold the largest values, rows without
    edges hold NaN and infinities, padding behind a passage held NaN before."""
    H, Ls = 4, [45, 64, 70]
    x = Held(B, Ls, H, H, D, 43)
    x.K, x.V = x.K.clone(), x.V.clone()
    x.K[45:109] = math.inf
    x.V[45:109] = -math.inf
    x.K[46] = -math.inf
    x.store.data.fill_(0xFF)
    x.write(B)
    x.off, x.po, x.pb = cum(Ls * nq), dev(cum(Ls * nq)), dev(np.tile(x.blocks, nq))
    Q = rows_of(6, H, D, 44)
    Q[2], Q[4] = math.nan, math.inf
    Q[5, 0, 0] = 2.0 ** 120                     # adjacent, but to nothing of that size
    nb = [[0], [0, 2], [], [2], [], []]
    O, lse = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [6] * nq, [3] * nq, 0.2, o_f32)
    torch.cuda.synchronize()
    O, lse = O.view(nq, 6, H, D), lse.view(nq, 6, H)
    assert (O == O[:1]).all() and (lse == lse[:1]).all()
    ref = reference(Q.double().numpy(), *x.held(cum(Ls)), nb, [6], [3], cum(Ls), 0.2, 1, o_f32)
    check(O[0], lse[0], ref, o_f32, "behind the mask")


# ---------------------------------------------------------------------------
# Together

def the_way(B, db, store, pb, packed, M, W_out, ws):
    """Pruning, the passages into the store, attention over it with rows in place,
    the output projection with the kept tokens' skip connection, a perceptron."""
    idx, _, _ = B.prune_topk(db, want_scores=False, want_rows=False)
    keys = B.quantize_passages(db.p, store, db.Kh, db.Vh, db.passage_offsets, pb, want_keys=True)
    O, lse = B.bipartite_xattn_quant(db.p, store, db.V, db.kept_offsets, db.passage_offsets, pb,
                                     db.query_passages, kept_idx=idx, passage_keys=keys,
                                     workspace=ws)
    d = db.p.d
    Y = B.gather_dense(db.p, O, packed[0], d, db.kept_offsets, residual=db.V, residual_idx=idx)
    h = B.gather_dense(db.p, Y, packed[1], M, activation="gelu")
    return idx, keys, O, lse, Y, h


@pytest.mark.parametrize("n_q", [1, 3, 20])
def test_the_way_of_a_question(B, n_q):
    batch = wls.make_batch("llava_bf16", 4, B=n_q)
    db = B.to_device(batch)
    p, d, M = db.p, db.p.d, 1408
    blocks, end = B.passage_blocks(batch.passage_offsets)
    store = B.new_kv_store(p.H, p.d_h, end)
    pb = dev(blocks)
    g = torch.Generator(device="cuda").manual_seed(45)
    W1 = (torch.randn(d, d, generator=g, device="cuda") / math.sqrt(d)).bfloat16()
    W2 = (torch.randn(M, d, generator=g, device="cuda") / math.sqrt(d)).bfloat16()
    packed = B.pack_dense(p, W1), B.pack_dense(p, W2)
    ws = torch.empty(B.workspace_bytes_quant(p, store), dtype=torch.uint8, device="cuda")

    def call():
        return the_way(B, db, store, pb, packed, M, None, ws)
    idx, keys, O, lse, Y, h = call()
    torch.cuda.synchronize()
    # the steps, each from the step before it as the device left it
    rows = torch.cat([batch.V[b][idx[a:c].long().cpu()] for b, (a, c) in
                      enumerate(zip(batch.kept_offsets[:-1], batch.kept_offsets[1:]))])
    Kd, Vd = B.dequantize_passages(p, store, db.passage_offsets, pb)
    Kd, Vd = Kd.cpu().double().numpy(), Vd.cpu().double().numpy()
    a, b = int(batch.passage_offsets[0]), int(batch.passage_offsets[1])
    held = orc.held_passage(batch.Kh[a:b, :1].double().numpy(), batch.Vh[a:b, :1].double().numpy())
    assert np.array_equal(Kd[a:b, :1], held[0]) and np.array_equal(Vd[a:b, :1], held[1])
    k0, P0 = int(batch.kept_offsets[1]), int(batch.query_passages[1])
    adj = orc.bsca_edges(orc.cosine_matrix(rows[:k0].double().numpy(),
                                           keys[:P0].cpu().double().numpy()), 4.0)
    nb = [np.nonzero(r)[0].tolist() for r in adj]
    ref = reference(rows[:k0].view(-1, p.H, p.d_h).double().numpy(), Kd, Vd, nb, [k0], [P0],
                    np.asarray(batch.passage_offsets), batch.wl.scale, 1)
    check(O[:k0], lse[:k0], ref, False, "the way")
    Od, Yd = O.reshape(-1, d).double(), Y.double()
    want = Od @ W1.double().t() + rows.cuda().double()
    mag = Od.abs() @ W1.double().abs().t()
    assert ((Yd - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -24 * (d + 3) * mag).all()
    want = act64(Yd @ W2.double().t(), "gelu")
    mag = Yd.abs() @ W2.double().abs().t()
    assert ((h.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * (want.abs() + 2.0 ** -4)
            + 1.13 * 2.0 ** -24 * (d + 3) * mag).all()
    check_replays(call)


@pytest.mark.parametrize("ks,Ps,L,D,H,Hkv", [([1], [4], 2000, 128, 4, 1),       # split, joined
                                             ([40, 3], [3, 4], 90, 64, 4, 4),   # row tiles
                                             ([9] * 200, [3] * 200, 70, 64, 4, 4)])  # many items
@pytest.mark.parametrize("o_f32", [False, True])
def test_capture_of_each_form(B, ks, Ps, L, D, H, Hkv, o_f32):
    x = Held(B, [L] * sum(Ps), H, Hkv, D, 46)
    keys = x.write(B, want_keys=True)
    Q = rows_of(sum(ks), H, D, 47).cuda()
    p = B.make_problem("bf16", B=len(ks), d=H * D, H=H, d_h=D, kept_offsets=cum(ks),
                       passage_offsets=x.off, query_passages=cum(Ps), avg_degree=2.0, o_f32=o_f32)
    ws = torch.empty(B.workspace_bytes_quant(p, x.store), dtype=torch.uint8, device="cuda")
    args = (dev(cum(ks)), x.po, x.pb, dev(cum(Ps)))
    nb = random_graph(ks, Ps, 48)
    q = B.make_problem("bf16", B=len(ks), d=H * D, H=H, d_h=D, kept_offsets=cum(ks),
                       passage_offsets=x.off, query_passages=cum(Ps), o_f32=o_f32,
                       total_edges=sum(map(len, nb)))
    graph = dev(cum([len(r) for r in nb])), dev([j for r in nb for j in r] or [0])[:q.total_edges]
    K, V = x.K.cuda(), x.V.cuda()

    def call():
        again = B.quantize_passages(x.p, x.store, K, V, x.po, x.pb, want_keys=True)
        a = B.bipartite_xattn_quant(p, x.store, Q, *args, passage_keys=again, workspace=ws)
        b = B.bipartite_xattn_quant(q, x.store, Q, *args, edges=graph, workspace=ws)
        return (again,) + a + b + B.dequantize_passages(x.p, x.store, x.po, x.pb)
    assert torch.equal(call()[0], keys)
    check_replays(call)


@pytest.mark.parametrize("M,d,d_out", [(5, 8192, 264), (20, 64, 72), (150, 8192, 264),
                                       (150, 96, 264), (1000, 64, 2048)])
def test_capture_of_the_layer(B, M, d, d_out):
    """Few rows and tiles, with a shared contraction and without."""
    g = torch.Generator(device="cuda").manual_seed(49)
    xr = torch.randn(M, d, generator=g, device="cuda").bfloat16()
    W = (torch.randn(d_out, d, generator=g, device="cuda") / math.sqrt(d)).bfloat16()
    R = torch.randn(M, d_out, generator=g, device="cuda").bfloat16()
    p = B.make_problem("bf16", B=1, d=d, kept_offsets=[0, M])
    ws = torch.empty(max(B.workspace_bytes_dense(p, d_out), 16), dtype=torch.uint8, device="cuda")

    def call():
        packed = B.pack_dense(p, W)
        return packed, B.gather_dense(p, xr, packed, d_out, activation="silu", residual=R,
                                      workspace=ws)
    check_replays(call)


def test_two_graphs_at_once(B):
    """Two captured calls over one store, each with its own workspace, replayed on
    two streams at once."""
    D, H, Ls = 128, 4, [900, 700, 1200]
    x = Held(B, Ls, H, 1, D, 50)
    keys = x.write(B, want_keys=True)
    d_out = 264
    p = B.make_problem("bf16", B=1, d=H * D, H=H, d_h=D, kept_offsets=[0, 3],
                       passage_offsets=x.off, query_passages=[0, 3], avg_degree=2.0)
    g = torch.Generator(device="cuda").manual_seed(51)
    W = (torch.randn(d_out, H * D, generator=g, device="cuda") / 16).bfloat16()
    packed = B.pack_dense(p, W)
    args = (dev([0, 3]), x.po, x.pb, dev([0, 3]))
    made = []
    for i in range(2):
        Q = rows_of(3, H, D, 52 + i).cuda()
        ws = torch.empty(B.workspace_bytes_quant(p, x.store), dtype=torch.uint8, device="cuda")
        wd = torch.empty(max(B.workspace_bytes_dense(p, d_out), 16), dtype=torch.uint8,
                         device="cuda")

        def call(Q=Q, ws=ws, wd=wd):
            O, lse = B.bipartite_xattn_quant(p, x.store, Q, *args, passage_keys=keys,
                                             workspace=ws)
            return O, lse, B.gather_dense(p, O, packed, d_out, workspace=wd)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = call()
        made.append((s, graph, out, want, call))            # (the call owns its tensors)
    assert not torch.equal(made[0][3][0], made[1][3][0])
    for _ in range(3):
        torch.cuda.synchronize()
        for s, graph, *_ in made:
            with torch.cuda.stream(s):
                for _ in range(4):
                    graph.replay()
        torch.cuda.synchronize()
        for _, _, out, want, _ in made:
            for a, b in zip(out, want):
                assert torch.equal(a, b)


def test_tensors_of_another_device_are_refused(B, monkeypatch):
    x = Held(B, [40], 2, 2, 64, 53)
    K, V = x.K.cuda(), x.V.cuda()
    p = B.make_problem("bf16", B=1, d=128, H=2, d_h=64, kept_offsets=[0, 4],
                       passage_offsets=x.off, query_passages=[0, 1], total_edges=4)
    Q, O = rows_of(4, 2, 64, 54).cuda(), torch.empty(4, 2, 64, device="cuda").bfloat16()
    ko, qp = dev([0, 4]), dev([0, 1])
    graph = dev([0, 1, 2, 3, 4]), dev([0, 0, 0, 0])
    W = torch.zeros(8, 128, dtype=torch.bfloat16, device="cuda")
    packed = B.pack_dense(p, W)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: B.quantize_passages(x.p, x.store, K, V, x.po, x.pb),
                 lambda: B.dequantize_passages(x.p, x.store, x.po, x.pb, (K, V)),
                 lambda: B.bipartite_xattn_quant(p, x.store, Q, ko, x.po, x.pb, qp, edges=graph,
                                                 out=(O, None), workspace=ws),
                 lambda: B.skip_pack_dense(p, W, packed),
                 lambda: B.gather_dense(p, Q, packed, 8, workspace=ws)):
        with pytest.raises(ValueError, match="device"):
            call()


@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("e", [15.0, 24.0, 29.5])
def test_many_small_weights(B, nq, D, e):
    """A token of weight 1 and value 0, 4000 of weight 2^-e and value 1 (all held as
    they are): no weight is lost, each off by 2^-11 of itself or 2^-32 of the largest
    (and its exponent by the float32 logit, 2^-22 e), the result by its own half step."""
    L, H = 4001, 4
    x = Held(B, [L], H, H, D, 55)
    x.K, x.V = torch.zeros_like(x.K), torch.ones_like(x.V)
    x.K[1:, :, 3] = -6.0
    x.V[0] = 0.0
    x.write(B)
    x.off, x.po, x.pb = cum([L] * nq), dev(cum([L] * nq)), dev(np.tile(x.blocks, nq))
    Q = torch.zeros(2, H, D).bfloat16()
    Q[:, :, 3] = 1.0
    O, lse = attend(B, x, Q.repeat(nq, 1, 1), [[0]] * (2 * nq), [2] * nq, [1] * nq,
                    e * math.log(2) / 6)
    torch.cuda.synchronize()
    s = 4000 * 2.0 ** -e
    want = s / (1 + s)
    err = (O.double() - want).abs().max().item()
    say(f"small weights e={e} D={D}: relative error {err / want:.2e}")
    assert err <= want * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -22 * e) + 4000 * 2.0 ** -32
    assert (lse.double() - math.log1p(s)).abs().max().item() <= 2.0 ** -20


def test_unknown_activation_is_refused(B):
    p = B.make_problem("bf16", B=1, d=64, kept_offsets=[0, 1])
    W = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="activation"):
        B.gather_dense(p, W[:1], B.pack_dense(p, W), 8, activation="tanh")


@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("o_f32", [False, True])
def test_the_largest_values_do_not_overflow(B, nq, D, o_f32):
    """Values near the largest held ones: the result is one of their averages."""
    H, Ls = 4, [300, 40]
    x = Held(B, Ls, H, H, D, 56, make=None)
    x.V = (x.V.float() * 2.0 ** 124).clamp(-2.0 ** 127, 2.0 ** 127).to(x.dt)
    x.write(B)
    x.off, x.po, x.pb = cum(Ls * nq), dev(cum(Ls * nq)), dev(np.tile(x.blocks, nq))
    Q = rows_of(5, H, D, 57)
    nb = [[0, 1], [1], [], [0], [0, 1]]
    O, lse = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [5] * nq, [2] * nq, 0.05, o_f32)
    torch.cuda.synchronize()
    O, lse = O.view(nq, 5, H, D), lse.view(nq, 5, H)
    assert (O == O[:1]).all() and (lse == lse[:1]).all()
    ref = reference(Q.double().numpy(), *x.held(cum(Ls)), nb, [5], [2], cum(Ls), 0.05, 1, o_f32)
    check(O[0], lse[0], ref, o_f32, "largest values")


def test_outputs_given_without_lse(B):
    x = Held(B, [40, 70], 2, 2, 64, 58)
    x.write(B)
    Q, nb = rows_of(6, 2, 64, 59), random_graph([6], [2], 60)
    O = torch.full((9, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got, none = attend(B, x, Q, nb, [6], [2], 0.2, out=(O, None))
    want, _ = attend(B, x, Q, nb, [6], [2], 0.2)
    torch.cuda.synchronize()
    assert none is None and torch.equal(got, want) and (O[6:] == 7.0).all()
