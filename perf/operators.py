"""Timed cases of the operators around a store of passages held in 4 bits: the
store written and read back, the bipartite attention over it, and the matrix
product with bias, activation and residual that follows the attention.

A case is a dict of plain values.  ``kind`` names the calls of one pass:

  quant   quantize_passages of a batch of passages into the store, then
          dequantize_passages of the same (the values that the store holds)
  attn    bipartite_xattn_quant: kept rows over the passages of the store, on
          a given graph or one built from the passage keys
  dense   gather_dense: act(W x + b) + residual of a batch of rows

``run`` makes these calls where ``own`` is set, and computes the same from
elementary operations otherwise.  The store's format is that of skip.h: blocks
of 32 values (32 features of a token's key, 32 tokens of a value feature), each
value one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, times its block's power of
two.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"

# quant, attn: heads (query) over heads_kv of d_h; P passages of L_lo..L_hi
# tokens for each of B questions, from a pool of `pool` stored passages (0: each
# its own); k kept rows a question, ragged: k and P over a quarter to two times;
# graph "given" (random neighbours, some rows without any), "complete" (given,
# every pair) or "built" (from the keys, by `degree`); index: rows read from
# [B][N][d] through the kept indices.  dense: M rows (per question k of N with
# index), d -> d_out.
DEFAULTS = dict(kind="attn", dtype="bf16", B=1, N=576, heads=16, heads_kv=16, d_h=64, k=96, P=5,
                L_lo=128, L_hi=128, pool=0, ragged=False, mix=1, graph="given", degree=4.0,
                index=False, o_f32=False, d=1024, d_out=1024, bias=True, act="none",
                residual=True)


def _case(**kw):
    return {**DEFAULTS, **kw}


def listed():
    return [
        # one short passage taken into the store: launches and latency
        _case(name="quant_one", kind="quant", heads=4, heads_kv=4, P=1, L_lo=61, L_hi=61),
        # the passages of a benchmark batch (highres_bf16)
        _case(name="quant_batch", kind="quant", B=16, heads=32, heads_kv=32, d_h=128, P=10,
              L_lo=256, L_hi=256),
        # float32 passages of any length, fewer key heads than query heads
        _case(name="quant_f32_ragged", kind="quant", dtype="f32", B=4, heads=32, heads_kv=8,
              d_h=128, P=20, L_lo=37, L_hi=301, mix=5),
        # one row of one question: the smallest call
        _case(name="attn_one_row", k=1, L_lo=61, L_hi=187, graph="complete", mix=2),
        # single rows over long stored documents, key heads shared by four
        _case(name="attn_rows_long", B=4, heads=32, heads_kv=8, d_h=128, k=1, P=20, L_lo=512,
              L_hi=2048, graph="complete", mix=3),
        # a small serving batch (llava_bf16), the graph from the keys
        _case(name="attn_llava", B=8, graph="built"),
        # the benchmark batch (highres_bf16)
        _case(name="attn_highres", B=16, N=2304, heads=32, heads_kv=32, d_h=128, k=192, P=10,
              L_lo=256, L_hi=256),
        # mixed difficulty over a shared pool of passages of any length, grouped
        # heads, rows in place, the graph from the keys
        _case(name="attn_grouped_mixed", B=24, N=2304, heads=32, heads_kv=8, d_h=128, k=167, P=9,
              L_lo=37, L_hi=301, pool=61, ragged=True, mix=4, graph="built", index=True),
        # one row through an output projection: latency
        _case(name="dense_one", kind="dense", k=1, d=1024, d_out=1024),
        # the visual projector's first layer on 8 images of 577 patches
        _case(name="dense_patches", kind="dense", B=8, k=577, d=1408, d_out=4096, act="gelu",
              residual=False),
        # the attention's output projection with the kept tokens' skip connection
        _case(name="dense_output", kind="dense", B=16, N=2304, k=193, d=4096, d_out=4096,
              bias=False, index=True),
        # a perceptron's second layer of few rows, float output, odd width
        _case(name="dense_down", kind="dense", B=3, k=97, d=16384, d_out=4104, act="silu",
              o_f32=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ranges: passages of 1..2048 tokens, 1..24 questions
    of 1..384 rows, products of 1..5000 rows, 256..16384 columns in, 64..8192
    out."""
    kind = rng.choice(["quant", "attn", "attn", "attn", "dense", "dense"])
    top = {"bytes": 0.0, "flops": 0.0}
    for c in listed():
        if c["kind"] == kind:
            w = work(c)
            top = {m: max(top[m], w[m]) for m in top}
    while True:
        c = _case(kind=kind, mix=rng.randint(1, 10 ** 6))
        if kind == "dense":
            c.update(B=rng.choice([1, 2, 5, 8]), k=_log_int(rng, 1, 600),
                     d=32 * _log_int(rng, 8, 512), d_out=8 * _log_int(rng, 8, 1024),
                     bias=rng.random() < 0.7, act=rng.choice(["none", "relu", "gelu", "silu"]),
                     residual=rng.random() < 0.7, index=rng.random() < 0.3,
                     o_f32=rng.random() < 0.25)
            c["N"] = c["k"] + rng.randint(0, 900)
        else:
            H, G, d_h = rng.choice([(4, 1, 64), (16, 1, 64), (16, 4, 64), (12, 3, 64), (8, 1, 128),
                                    (32, 1, 128), (32, 4, 128), (16, 2, 128), (32, 32, 128)])
            L = _log_int(rng, 1, 2048)
            c.update(heads=H, heads_kv=H // G, d_h=d_h, B=_log_int(rng, 1, 24),
                     P=_log_int(rng, 1, 20), L_lo=max(1, L // rng.choice([1, 2, 5])), L_hi=L)
            if kind == "quant":
                c.update(dtype=rng.choice(["bf16", "bf16", "f32"]))
            else:
                c.update(k=_log_int(rng, 1, 384), pool=rng.choice([0, 0, 7, 40]),
                         ragged=rng.random() < 0.5, degree=rng.choice([4.0, 4.0, 2.0, 1.0, 6.5]),
                         graph=rng.choice(["given", "complete", "built", "built"]),
                         index=rng.random() < 0.3, o_f32=rng.random() < 0.2)
                c["N"] = 2 * c["k"] + rng.randint(0, 2304)
        w = work(c)
        if w["bytes"] <= top["bytes"] and w["flops"] <= top["flops"]:
            return c


# ---------------------------------------------------------------------------
# Shapes

def _shape(c):
    """(rows per question, passages per question, stored passage of each, tokens
    of each stored passage)."""
    rng = random.Random(c["mix"])
    ks, Ps = [], []
    for _ in range(c["B"]):
        m = rng.choice((0.25, 0.5, 1, 2)) if c["ragged"] else 1
        n = rng.choice((0.25, 0.5, 1, 2)) if c["ragged"] else 1
        ks.append(max(1, min(c["N"], int(c["k"] * m))) if c["kind"] == "attn" else c["k"])
        Ps.append(max(1, min(20, int(c["P"] * n))))
    total = sum(Ps)
    stored = c["pool"] or total
    Ls = [rng.randint(c["L_lo"], c["L_hi"]) for _ in range(stored)]
    ids = [rng.randrange(stored) for _ in range(total)] if c["pool"] else list(range(total))
    return ks, Ps, ids, Ls


def _graph(c, ks, Ps):
    """Given neighbours: ascending passages of every kept row."""
    rng = random.Random(c["mix"] + 1)
    rows = []
    for k, P in zip(ks, Ps):
        for _ in range(k):
            n = P if c["graph"] == "complete" else min(P, rng.choice((0, 2, 3, 4, 4, 5, 5, 8)))
            rows.append(sorted(rng.sample(range(P), n)))
    return rows


def _cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int32)


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _blocks(Ls, mix):
    """First block of every stored passage, placed in any order with gaps, as a
    store that other passages came to and left."""
    rng = random.Random(mix + 2)
    order = list(range(len(Ls)))
    rng.shuffle(order)
    first, at = [0] * len(Ls), rng.randint(0, 3)
    for i in order:
        first[i] = at
        at += (Ls[i] + 31) // 32 + rng.choice((0, 0, 1))
    return first, at


def work(case):
    """Bytes and operations one pass cannot do without."""
    c = case
    if c["kind"] == "dense":
        M, o = c["B"] * c["k"], 4 if c["o_f32"] else 2
        n = M * c["d"] * 2 + c["d"] * c["d_out"] * 2 + M * c["d_out"] * o
        n += c["d_out"] * 4 * c["bias"] + M * c["d_out"] * 2 * c["residual"] + 4 * M * c["index"]
        return {"bytes": float(n), "flops": 2.0 * M * c["d"] * c["d_out"]}
    ks, Ps, ids, Ls = _shape(c)
    hk, d_h, H = c["heads_kv"], c["d_h"], c["heads"]
    nblk = [(L + 31) // 32 for L in Ls]
    if c["kind"] == "quant":                 # read, written to the store, read there, written
        e = 4 if c["dtype"] == "f32" else 2
        n = 2 * (2 * sum(Ls) * hk * d_h * e) + 2 * sum(nblk) * hk * 34 * d_h
        return {"bytes": float(n), "flops": 0.0}
    # every stored passage that a row is linked to, once; rows, outputs, graph
    d = H * d_h
    n, edges_tok, at, r0 = 0, 0, 0, 0
    used = set()
    rows = _graph(c, ks, Ps) if c["graph"] != "built" else None
    for k, P in zip(ks, Ps):
        tok = [Ls[i] for i in ids[at:at + P]]
        if rows is not None:
            for nb in rows[r0:r0 + k]:
                edges_tok += sum(tok[j] for j in nb)
                used.update(ids[at + j] for j in nb)
        else:
            edges = min(k * P, math.ceil(c["degree"] * k))
            edges_tok += edges * sum(tok) / P
            used.update(ids[at:at + P])
        at += P
        r0 += k
    n += sum(nblk[i] for i in used) * hk * 34 * d_h
    n += sum(ks) * (d * 2 + d * (4 if c["o_f32"] else 2) + 4 * H)
    if rows is None:
        n += sum(Ps) * d * 4
    return {"bytes": float(n), "flops": 4.0 * edges_tok * H * d_h}


# ---------------------------------------------------------------------------
# The store's format, from elementary operations

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _codes(x):
    """Codes and scale bytes of blocks of 32 along the last axis (float32)."""
    amax = x.abs().amax(-1)
    bits = amax.view(torch.int32)
    s = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x600000).int()).clamp(1, 254)
    y = torch.ldexp(x.abs(), (127 - s)[..., None])
    code = torch.zeros_like(y, dtype=torch.uint8)
    for lim, even in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        code += (y >= lim if even else y > lim).to(torch.uint8)      # ties to the even code
    return code | (torch.signbit(x).to(torch.uint8) << 3), s.to(torch.uint8)


def _pairs(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _plan(Ls, first):
    """The blocks that passages take in the store, and for every token its slot
    among them."""
    blocks = [f + i for f, L in zip(first, Ls) for i in range((L + 31) // 32)]
    start = 32 * _cum([(L + 31) // 32 for L in Ls])
    where = np.concatenate([a + np.arange(L) for a, L in zip(start, Ls)])
    return (torch.tensor(blocks, dtype=torch.int64, device=DEV),
            torch.from_numpy(where.astype(np.int64)).to(DEV))


def _store(Kh, Vh, plan, data):
    """Writes passages into the store `data` [blocks][heads][34 d_h]."""
    _, hk, D = Kh.shape
    touched, where = plan
    pad = torch.zeros(2, touched.numel() * 32, hk, D, dtype=torch.float32, device=Kh.device)
    pad[0, where] = Kh.float()
    pad[1, where] = Vh.float()
    nb, C = touched.numel(), D // 32
    kc, ks = _codes(pad[0].view(nb, 2, 16, hk, C, 32))
    vc, vs = _codes(pad[1].view(nb, 32, hk, D).permute(0, 2, 3, 1).contiguous())
    data[touched] = torch.cat([
        _pairs(kc).permute(0, 3, 1, 4, 2, 5).reshape(nb, hk, 16 * D),
        _pairs(vc).reshape(nb, hk, 16 * D),
        ks.view(nb, 2, 16, hk, C // 2, 2).permute(0, 3, 5, 2, 1, 4).reshape(nb, hk, D),
        vs.view(nb, hk, C, 32).transpose(2, 3).reshape(nb, hk, D)], 2)


def _read(data, plan, D):
    """Keys and values of the plan's tokens, float32 [tokens][heads][d_h]."""
    touched, where = plan
    rec = data[touched]
    nb, hk, C = rec.shape[0], rec.shape[1], D // 32
    lut = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=data.device)

    def values(b, s):
        v = lut[torch.stack([b & 15, b >> 4], -1).flatten(-2).int()]
        return torch.ldexp(v, s.int()[..., None] - 127)
    k = rec[:, :, :16 * D].view(nb, hk, 2, C, 16, 16).permute(0, 2, 4, 1, 3, 5)
    v = rec[:, :, 16 * D:32 * D].view(nb, hk, D, 16)
    ks = rec[:, :, 32 * D:33 * D].view(nb, hk, 2, 16, 2, C // 2).permute(0, 4, 3, 1, 5, 2)
    vs = rec[:, :, 33 * D:].view(nb, hk, 32, C).transpose(2, 3).reshape(nb, hk, D)
    K = values(k, ks.reshape(nb, 2, 16, hk, C)).reshape(nb * 32, hk, D)
    V = values(v, vs).permute(0, 3, 1, 2).reshape(nb * 32, hk, D)
    return K[where], V[where]


# ---------------------------------------------------------------------------
# Inputs

def _inputs(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if c["kind"] == "dense":
        M, d, n = c["B"] * c["k"], c["d"], c["d_out"]
        x = {"rows": torch.randn(M, d, generator=g, device=DEV).bfloat16(),
             "W": (torch.randn(n, d, generator=g, device=DEV) / math.sqrt(d)).bfloat16(),
             "b": 0.2 * torch.randn(n, generator=g, device=DEV) if c["bias"] else None,
             "R": None, "idx": None}
        if c["residual"]:
            r = c["B"] * c["N"] if c["index"] else M
            x["R"] = torch.randn(r, n, generator=g, device=DEV).bfloat16()
            if c["index"]:
                x["idx"] = _indices(c, [c["k"]] * c["B"], g)
        return x
    ks, Ps, ids, Ls = _shape(c)
    hk, D, dt = c["heads_kv"], c["d_h"], _dtype(c)
    n, d = sum(Ls), c["heads"] * c["d_h"]
    mu = 0.5 * torch.randn(len(Ls), hk * D, generator=g, device=DEV)
    owner = torch.repeat_interleave(torch.arange(len(Ls), device=DEV),
                                    torch.tensor(Ls, device=DEV))
    Kh = torch.empty(n, hk * D, dtype=dt, device=DEV)
    Vh = torch.empty(n, hk * D, dtype=dt, device=DEV)
    step = max(1, (1 << 26) // (hk * D))
    for i in range(0, n, step):
        m = min(step, n - i)
        Kh[i:i + m] = mu[owner[i:i + m]] + torch.randn(m, hk * D, generator=g, device=DEV)
        Vh[i:i + m] = torch.randn(m, hk * D, generator=g, device=DEV)
    x = {"Kh": Kh.view(n, hk, D), "Vh": Vh.view(n, hk, D)}
    if c["kind"] == "quant":
        return x
    # kept rows of width 1/sqrt(d) an element, as the workloads draw visual tokens
    M = c["B"] * c["N"] if c["index"] else sum(ks)
    x["Q"] = (torch.randn(M, d, generator=g, device=DEV) / math.sqrt(d)).bfloat16()
    x["idx"] = _indices(c, ks, g) if c["index"] else None
    # the keys that were kept when the passages were encoded: their mean key, one
    # copy a query head
    sums = torch.zeros(len(Ls), hk * D, device=DEV).index_add_(0, owner, Kh.float())
    mean = (sums / torch.tensor(Ls, device=DEV)[:, None]).view(-1, hk, D)
    mean = mean.repeat_interleave(c["heads"] // hk, 1).reshape(-1, d)
    x["keys"] = mean[torch.tensor(ids, device=DEV)].contiguous() if c["graph"] == "built" else None
    return x


def _indices(c, ks, g):
    """Kept tokens of each question, ascending."""
    return torch.cat([torch.randperm(c["N"], generator=g, device=DEV)[:k].sort().values
                      for k in ks]).int()


def prepare(case, seed):
    c = case
    s = {"c": c, **_inputs(c, seed)}
    dev = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    if own:
        from paper_2607_25422_amd import binding as B
        s["B"] = B
    if c["kind"] == "dense":
        s["out"] = torch.empty(c["B"] * c["k"], c["d_out"], device=DEV,
                               dtype=torch.float32 if c["o_f32"] else torch.bfloat16)
        if c["index"] and c["residual"]:
            s["src"] = (torch.arange(c["B"], device=DEV).repeat_interleave(c["k"]) * c["N"] +
                        s["idx"].long())
        if own:
            off = _cum([c["k"]] * c["B"])
            s["p"] = B.make_problem("bf16", B=c["B"], N=c["N"], d=c["d"], kept_offsets=off)
            s["off"] = dev(off)
            s["packed"] = B.pack_dense(s["p"], s["W"])       # weights are laid out once
        return s
    ks, Ps, ids, Ls = _shape(c)
    first, n_blocks = _blocks(Ls, c["mix"])
    hk, D = c["heads_kv"], c["d_h"]
    s["plan"] = _plan(Ls, first)
    s["data"] = torch.zeros(n_blocks, hk, 34 * D, dtype=torch.uint8, device=DEV)
    common = dict(d=c["heads"] * D, H=c["heads"], d_h=D, o_f32=c["o_f32"])
    if c["kind"] == "quant":
        if own:
            po = _cum(Ls)
            s["p"] = B.make_problem(c["dtype"], B=1, passage_offsets=po,
                                    query_passages=[0, len(Ls)], **common)
            s["po"], s["pb"] = dev(po), dev(first)
            s["store"] = B.KvStore(s["data"], hk, n_blocks)
            s["out"] = torch.empty_like(s["Kh"]), torch.empty_like(s["Vh"])
        return s
    _store(s.pop("Kh"), s.pop("Vh"), s["plan"], s["data"])          # filled before
    s["scale"] = math.sqrt(c["heads"])          # sqrt(d) / sqrt(d_h) for rows of width 1/sqrt(d)
    ko, po, qp = _cum(ks), _cum([Ls[i] for i in ids]), _cum(Ps)
    at = _cum(Ls)
    s["host"] = ko, qp
    s["tok"] = [[(int(at[i]), int(at[i + 1])) for i in ids[qp[b]:qp[b + 1]]]
                for b in range(c["B"])]
    if c["index"]:
        s["src"] = torch.repeat_interleave(torch.arange(c["B"], device=DEV), dev(ks)) * c["N"]
        s["src"] = s["src"] + s["idx"].long()
    s["rowptr"] = s["col"] = None
    if c["graph"] != "built":
        rows = _graph(c, ks, Ps)
        s["host_rowptr"] = _cum([len(r) for r in rows])
        s["rowptr"] = dev(s["host_rowptr"])
        s["col"] = dev([j for r in rows for j in r] or [0])[:sum(len(r) for r in rows)]
    d = c["heads"] * D
    s["O"] = torch.empty(sum(ks), c["heads"], D, device=DEV,
                         dtype=torch.float32 if c["o_f32"] else torch.bfloat16)
    s["lse"] = torch.empty(sum(ks), c["heads"], device=DEV)
    if own:
        s["p"] = B.make_problem("bf16", B=c["B"], N=c["N"], avg_degree=c["degree"],
                                sm_scale=s["scale"], kept_offsets=ko, passage_offsets=po,
                                query_passages=qp,
                                total_edges=0 if s["col"] is None else s["col"].numel(), **common)
        s["ko"], s["po"], s["qp"] = dev(ko), dev(po), dev(qp)
        s["pb"] = dev([first[i] for i in ids])
        s["store"] = B.KvStore(s["data"], hk, n_blocks)
        s["ws"] = torch.empty(B.workspace_bytes_quant(s["p"], s["store"]), dtype=torch.uint8,
                              device=DEV)
    return s


# ---------------------------------------------------------------------------
# One pass

def run(state):
    s = state
    return {"quant": _run_quant, "attn": _run_attn, "dense": _run_dense}[s["c"]["kind"]](s)


def _run_quant(s):
    if own:
        B = s["B"]
        B.quantize_passages(s["p"], s["store"], s["Kh"], s["Vh"], s["po"], s["pb"])
        return B.dequantize_passages(s["p"], s["store"], s["po"], s["pb"], out=s["out"])
    _store(s["Kh"], s["Vh"], s["plan"], s["data"])
    K, V = _read(s["data"], s["plan"], s["c"]["d_h"])
    return K.to(s["Kh"].dtype), V.to(s["Kh"].dtype)


def _adjacent(q, keys, degree):
    """Edges of one question: the ceil(degree * k) largest cosines of its pairs,
    ties to the lower pair (float64: a cut between neighbouring values)."""
    q, keys = q.double(), keys.double()
    k, P = q.shape[0], keys.shape[0]
    n = q.norm(dim=1)[:, None] * keys.norm(dim=1)[None]
    cos = torch.where(n > 0, (q @ keys.t()) / n.clamp_min(1e-300), torch.zeros_like(n)).flatten()
    E = min(k * P, math.ceil(degree * k))
    adj = torch.zeros(k * P, dtype=torch.bool, device=q.device)
    adj[torch.sort(cos, descending=True, stable=True).indices[:E]] = True
    return adj.view(k, P)


def _given(s, r0, r1, P):
    """Edges of one question from the graph's rows r0 .. r1 - 1."""
    a, b = int(s["host_rowptr"][r0]), int(s["host_rowptr"][r1])
    rp = s["rowptr"]
    adj = torch.zeros(r1 - r0, P, dtype=torch.bool, device=DEV)
    rows = torch.repeat_interleave(torch.arange(r1 - r0, device=DEV),
                                   (rp[r0 + 1:r1 + 1] - rp[r0:r1]).long(), output_size=b - a)
    adj[rows, s["col"][a:b].long()] = True
    return adj


def _run_attn(s):
    c = s["c"]
    if own:
        return s["B"].bipartite_xattn_quant(
            s["p"], s["store"], s["Q"], s["ko"], s["po"], s["pb"], s["qp"], kept_idx=s["idx"],
            passage_keys=s["keys"], edges=None if s["col"] is None else (s["rowptr"], s["col"]),
            out=(s["O"], s["lse"]), workspace=s["ws"])
    H, hk, D = c["heads"], c["heads_kv"], c["d_h"]
    K, V = _read(s["data"], s["plan"], D)
    Q = s["Q"][s["src"]] if c["index"] else s["Q"]
    ko, qp = s["host"]
    O, lse = s["O"], s["lse"]
    for b in range(c["B"]):
        r0, r1, tok = int(ko[b]), int(ko[b + 1]), s["tok"][b]
        q = Q[r0:r1]
        if s["col"] is None:
            adj = _adjacent(q, s["keys"][int(qp[b]):int(qp[b + 1])], c["degree"])
        else:
            adj = _given(s, r0, r1, len(tok))
        k = torch.cat([K[i:j] for i, j in tok]).permute(1, 2, 0)               # hk, D, n
        v = torch.cat([V[i:j] for i, j in tok]).transpose(0, 1)                # hk, n, D
        mask = torch.cat([adj[:, j:j + 1].expand(-1, e - a)
                          for j, (a, e) in enumerate(tok)], 1)
        q = q.float().view(r1 - r0, hk, H // hk, D).permute(1, 2, 0, 3).reshape(hk, -1, D)
        z = (q @ k * s["scale"]).view(hk, H // hk, r1 - r0, -1)
        z = z.masked_fill(~mask, float("-inf"))
        m = z.amax(-1, keepdim=True)
        m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
        p = torch.exp(z - m)
        l = p.sum(-1, keepdim=True)
        o = (p.view(hk, -1, p.shape[-1]) @ v).view(hk, H // hk, r1 - r0, D)
        o = torch.where(l > 0, o / l.clamp_min(1e-38), torch.zeros_like(o))
        O[r0:r1] = o.permute(2, 0, 1, 3).reshape(r1 - r0, H, D).to(O.dtype)
        lse[r0:r1] = (m + torch.log(l)).squeeze(-1).permute(2, 0, 1).reshape(r1 - r0, H)
    return O, lse


def _act(y, name, one):
    if name == "relu":
        return torch.where(y > 0, y, torch.zeros_like(y))
    if name == "gelu":
        return 0.5 * y * (one + torch.erf(y * math.sqrt(0.5)))
    if name == "silu":
        return y / (one + torch.exp(-y))
    return y


def _run_dense(s):
    c = s["c"]
    if own:
        return s["B"].gather_dense(s["p"], s["rows"], s["packed"], c["d_out"], s["off"],
                                   bias=s["b"], activation=c["act"], residual=s["R"],
                                   residual_idx=s["idx"], out=s["out"])
    y = s["rows"].float() @ s["W"].float().t()
    if s["b"] is not None:
        y = y + s["b"]
    y = _act(y, c["act"], 1.0)
    if s["R"] is not None:
        y = y + (s["R"][s["src"]] if c["index"] else s["R"]).float()
    return y.to(s["out"].dtype)


# ---------------------------------------------------------------------------
# From the definitions, in 64 bits

def _nearest(x):
    """What a block of 32 (last axis) is held as: the power of two and the
    nearest of the sixteen values, a tie to the neighbour of even position."""
    a = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(a.clamp_min(2.0 ** -200))) - 2
    e = torch.where(a > 7 * torch.exp2(e), e + 1, e)         # (log2 may sit a step off)
    e = torch.where(a <= 7 * torch.exp2(e - 1), e - 1, e).clamp(-126, 127)
    y = x.abs() / torch.exp2(e)
    grid = torch.tensor(_VALUES, dtype=torch.float64, device=x.device)
    up = torch.searchsorted(grid, y.contiguous()).clamp(1, 7)
    lo, hi = grid[up - 1], grid[up]
    take = (y - lo > hi - y) | ((y - lo == hi - y) & (up % 2 == 0))
    return torch.where(take, hi, lo) * torch.sign(x) * torch.exp2(e)


def _held(c, x, Ls):
    """Keys and values as held, float64, passage by passage."""
    hk, D = c["heads_kv"], c["d_h"]
    at = _cum(Ls)
    K = torch.empty(sum(Ls), hk, D, dtype=torch.float64, device=DEV)
    V = torch.empty_like(K)
    for i, L in enumerate(Ls):
        a, b, n = int(at[i]), int(at[i + 1]), (L + 31) // 32
        K[a:b] = _nearest(x["Kh"][a:b].double().view(L, hk, D // 32, 32)).view(L, hk, D)
        v = torch.zeros(n * 32, hk, D, dtype=torch.float64, device=DEV)
        v[:L] = x["Vh"][a:b].double()
        v = _nearest(v.view(n, 32, hk, D).permute(0, 2, 3, 1).contiguous())
        V[a:b] = v.permute(0, 3, 1, 2).reshape(n * 32, hk, D)[:L]
    return K, V


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    if c["kind"] == "dense":
        out = torch.empty(c["B"] * c["k"], c["d_out"], dtype=torch.float64, device=DEV)
        W = x["W"].double()
        for b in range(c["B"]):
            rows = slice(b * c["k"], (b + 1) * c["k"])
            y = torch.matmul(x["rows"][rows].double(), W.T)
            if x["b"] is not None:
                y += x["b"].double()
            if c["act"] == "relu":
                y = y.clamp_min(0)
            elif c["act"] == "gelu":
                y = y * torch.special.ndtr(y)
            elif c["act"] == "silu":
                y = y * torch.sigmoid(y)
            if x["R"] is not None:
                y += (x["R"][b * c["N"]:(b + 1) * c["N"]][x["idx"][rows].long()] if c["index"]
                      else x["R"][rows]).double()
            out[rows] = y
        return out
    ks, Ps, ids, Ls = _shape(c)
    K, V = _held(c, x, Ls)
    if c["kind"] == "quant":
        return K, V
    H, hk, D = c["heads"], c["heads_kv"], c["d_h"]
    G = H // hk
    at = _cum(Ls)
    O = torch.zeros(sum(ks), H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((sum(ks), H), float("-inf"), dtype=torch.float64, device=DEV)
    nb = _graph(c, ks, Ps) if c["graph"] != "built" else None
    r0 = p0 = 0
    for b, (k, P) in enumerate(zip(ks, Ps)):
        if c["index"]:
            q = x["Q"][b * c["N"] + x["idx"][r0:r0 + k].long()].double()
        else:
            q = x["Q"][r0:r0 + k].double()
        link = np.zeros((k, P), dtype=bool)
        if nb is not None:
            for i in range(k):
                link[i, nb[r0 + i]] = True
        else:
            key = x["keys"][p0:p0 + P].double().cpu().numpy()
            qn = q.cpu().numpy()
            n = np.linalg.norm(qn, axis=1)[:, None] * np.linalg.norm(key, axis=1)[None]
            cos = np.where(n > 0, qn @ key.T / np.where(n > 0, n, 1), 0.0).ravel()
            E = min(k * P, math.ceil(c["degree"] * k))
            link.reshape(-1)[np.lexsort((np.arange(k * P), -cos))[:E]] = True
        link = torch.from_numpy(link).to(DEV)
        q = q.view(k, hk, G, D)
        # passage by passage: sums against the running maximum of each row
        m = torch.full((k, H), float("-inf"), dtype=torch.float64, device=DEV)
        l = torch.zeros(k, H, dtype=torch.float64, device=DEV)
        o = torch.zeros(k, H, D, dtype=torch.float64, device=DEV)
        for j in range(P):
            rows = link[:, j].nonzero().flatten()
            if rows.numel() == 0:
                continue
            a, e = int(at[ids[p0 + j]]), int(at[ids[p0 + j] + 1])
            qq = q[rows].permute(1, 0, 2, 3).reshape(hk, -1, D)
            z = torch.matmul(qq, K[a:e].permute(1, 2, 0).contiguous()) * math.sqrt(H)
            z = z.view(hk, rows.numel(), G, e - a)
            top = z.amax(-1).permute(1, 0, 2).reshape(-1, H)
            mn = torch.maximum(m[rows], top)
            f = torch.exp(m[rows] - mn)
            w = torch.exp(z - mn.view(-1, hk, G).permute(1, 0, 2)[..., None])
            l[rows] = l[rows] * f + w.sum(-1).permute(1, 0, 2).reshape(-1, H)
            pv = torch.matmul(w.view(hk, -1, e - a), V[a:e].transpose(0, 1).contiguous())
            pv = pv.view(hk, rows.numel(), G, D).permute(1, 0, 2, 3).reshape(-1, H, D)
            o[rows] = o[rows] * f[..., None] + pv
            m[rows] = mn
        has = link.any(1)
        O[r0:r0 + k][has] = o[has] / l[has][..., None]
        lse[r0:r0 + k][has] = m[has] + torch.log(l[has])
        r0 += k
        p0 += P
    return O, lse
