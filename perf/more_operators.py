"""Timed cases of the operators around a paged cache of keys and values: new
tokens rotated and appended, attention of the new tokens over the cache with
prefixes that several sequences share, and attention over the pages that a score
selects for each new token.

A case is a dict of plain values.  ``kind`` names the calls of one pass:

  append  cache_append: queries and keys of the new tokens rotated by their
          positions, keys and values written into the pages, the pages' mean
          keys brought up to date
  attn    cache_attn: new tokens over the cache, causal; shared prefixes once
          for the sequences that share them
  pages   cache_select, then cache_attn_pages: for every new token and key head
          the pages of the largest <sum of the head group's queries, mean key>,
          and attention over those pages alone

``run`` makes these calls where ``own`` is set, and computes the same from
elementary operations otherwise.  Sequence b holds lens[b] tokens, the new ones
(rows row_offsets[b] .. row_offsets[b + 1] - 1) the last of them; token t lies in
page page_table[b][t // page], at t % page.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"

# B sequences of n_lo..n_hi new tokens after L_lo..L_hi earlier ones (0: none),
# for heads query heads over heads_kv key heads of d_h, in pages of `page` tokens.
# append: rows of dtype (packed: q, k and v of a token in one row of a projection's
# output), rotated by "halves" or "pairs" of `rot` features (0: not), by positions
# of their own (a kept visual token's place in its image) with `placed`.  attn: the
# sequences form `groups` equal runs whose first `prefix` tokens are shared (before
# the L earlier ones).  pages: n_sel pages for a token and key head, the n_first
# first and the n_last last always among them.
DEFAULTS = dict(kind="attn", dtype="bf16", B=1, heads=32, heads_kv=8, d_h=128, page=64, n_lo=1,
                n_hi=1, L_lo=0, L_hi=0, groups=0, prefix=0, o_f32=False, style="halves", rot=128,
                packed=True, placed=False, n_sel=0, n_first=1, n_last=1, mix=1)


def _case(**kw):
    return {**DEFAULTS, **kw}


def listed():
    return [
        # one token of one sequence: launches and latency
        _case(name="append_one", kind="append", heads=16, heads_kv=16, d_h=64, rot=64, L_lo=60,
              L_hi=60),
        # a serving batch, one token each
        _case(name="append_decode", kind="append", B=64, L_lo=100, L_hi=4000, mix=2),
        # the fused tokens and questions of a batch taken in: kept visual tokens with
        # the positions that they have in their image
        _case(name="append_prefill", kind="append", B=16, n_lo=224, n_hi=608, placed=True, mix=3),
        # float32 rows, each array on its own, part of the features rotated in pairs,
        # sequences of any length continued
        _case(name="append_f32_ragged", kind="append", dtype="f32", B=5, heads=12, heads_kv=3,
              d_h=64, page=32, n_lo=1, n_hi=333, L_lo=1, L_hi=700, style="pairs", rot=48,
              packed=False, mix=4),
        # one token over a short sequence: the smallest call
        _case(name="attn_one", heads=16, heads_kv=16, d_h=64, L_lo=60, L_hi=60),
        # a serving batch of mixed lengths, one token each, nothing shared
        _case(name="attn_decode", B=48, L_lo=300, L_hi=16384, mix=5),
        # answers sampled from four shared contexts (passages and kept tokens)
        _case(name="attn_shared", B=64, groups=4, prefix=8217, L_lo=1, L_hi=500, mix=6),
        # a batch of prompts, causal
        _case(name="attn_prefill", B=4, n_lo=1024, n_hi=4096, mix=7),
        # the next pieces of long prompts over a common context, float32 output
        _case(name="attn_chunk", B=6, heads=16, heads_kv=16, d_h=64, page=32, n_lo=97, n_hi=131,
              groups=2, prefix=3001, L_lo=1, L_hi=900, o_f32=True, mix=8),
        # one token of one sequence, few pages
        _case(name="pages_one", kind="pages", L_lo=4000, L_hi=4000, n_sel=8),
        # a serving batch of long sequences, one token each
        _case(name="pages_decode", kind="pages", B=32, L_lo=8000, L_hi=65000, n_sel=32, n_last=2,
              mix=9),
        # several tokens a sequence (drafts to be checked), every head its own keys
        _case(name="pages_rows", kind="pages", B=4, heads=16, heads_kv=16, d_h=64, page=32, n_lo=5,
              n_hi=61, L_lo=500, L_hi=6000, n_sel=17, n_last=2, o_f32=True, mix=10),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ranges: 1..64 sequences of 1 to tens of thousands of
    tokens, 1..4096 new tokens each, pages of 32..256 tokens."""
    kind = rng.choice(["append", "append", "attn", "attn", "attn", "pages", "pages"])
    top = {"bytes": 0.0, "flops": 0.0, "held": 0.0}
    for c in listed():
        if c["kind"] == kind:
            w = {**work(c), "held": _held(c)}
            top = {m: max(top[m], w[m]) for m in top}
    while True:
        c = _case(kind=kind, mix=rng.randint(1, 10 ** 6))
        H, G, d_h = rng.choice([(16, 1, 64), (12, 4, 64), (32, 4, 64), (32, 1, 128), (32, 4, 128),
                                (24, 8, 128), (16, 16, 128), (32, 32, 128), (15, 5, 128)])
        c.update(heads=H, heads_kv=H // G, d_h=d_h, page=rng.choice([32, 64, 64, 128, 256]),
                 B=_log_int(rng, 1, 64))
        if kind == "append":
            n, L = _log_int(rng, 1, 1500), _log_int(rng, 1, 4000)
            c.update(n_lo=max(1, n // rng.choice([1, 2, 7])), n_hi=n, L_lo=rng.choice([0, 1, L]),
                     L_hi=L, dtype=rng.choice(["bf16", "bf16", "f32"]),
                     style=rng.choice(["halves", "pairs"]),
                     rot=rng.choice([d_h, d_h, d_h // 2, 16 * rng.randint(0, d_h // 16)]),
                     packed=rng.random() < 0.6, placed=rng.random() < 0.3)
        elif kind == "attn":
            n = rng.choice([1, 1, _log_int(rng, 1, 16), _log_int(rng, 16, 4096)])
            L = _log_int(rng, 1, 16384)
            c.update(n_lo=max(1, n // rng.choice([1, 2, 5])), n_hi=n, L_lo=rng.choice([0, 1, L]),
                     L_hi=L, o_f32=rng.random() < 0.25)
            if rng.random() < 0.5 and c["B"] > 1:
                c.update(groups=rng.randint(1, c["B"]), prefix=_log_int(rng, 1, 10000))
        else:
            n, L = rng.choice([1, 1, _log_int(rng, 1, 64)]), _log_int(rng, 1, 65000)
            c.update(n_lo=max(1, n // rng.choice([1, 3])), n_hi=n, L_lo=max(1, L // 8), L_hi=L,
                     n_sel=_log_int(rng, 2, 64), o_f32=rng.random() < 0.25)
            c["n_last"] = rng.randint(1, min(4, c["n_sel"]))
            c["n_first"] = rng.randint(0, min(2, c["n_sel"] - c["n_last"]))
        w = {**work(c), "held": _held(c)}
        if all(w[m] <= top[m] for m in top):
            return c


# ---------------------------------------------------------------------------
# Shapes

def _shape(c):
    """(new tokens, tokens held, shared prefix, group) of every sequence."""
    rng = random.Random(c["mix"])
    out = []
    for b in range(c["B"]):
        n = rng.randint(c["n_lo"], c["n_hi"])
        L = _log_int(rng, max(1, c["L_lo"]), c["L_hi"]) if c["L_hi"] else 0
        g = b * c["groups"] // c["B"] if c["groups"] else -1
        P = c["prefix"] if g >= 0 else 0
        out.append((n, P + L + n, P, g))
    return out


def _tables(c, shape):
    """Physical pages of every sequence, in any order; whole pages of a shared
    prefix are the same ones; (table, pages, [(page of the group's first sequence,
    own page, tokens)] of prefixes that end inside a page)."""
    page = c["page"]
    need = [-(-ln // page) for _, ln, _, _ in shape]
    rng = random.Random(c["mix"] + 1)
    own_first = {}
    total, logical, shared = 0, [], []
    for b, (_, ln, P, g) in enumerate(shape):
        first = own_first.setdefault(g, b) if g >= 0 else b
        keep = P // page if first != b else 0
        ids = list(logical[first][:keep]) if keep else []
        new = list(range(total, total + need[b] - keep))
        total += len(new)
        ids += new
        if first != b and P % page:
            shared.append((logical[first][keep], ids[keep], P % page))
        logical.append(ids)
    pages = total + 3
    place = list(range(pages))
    rng.shuffle(place)
    table = np.full((c["B"], max(need) + rng.randint(0, 2)), -1, dtype=np.int32)
    for b, ids in enumerate(logical):
        table[b, :len(ids)] = [place[i] for i in ids]
    return table, pages, [(place[a], place[i], t) for a, i, t in shared]


def _cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int32)


def _pairs(n, ln):
    """Pairs of a new token and a token that it sees."""
    return n * (ln - n) + n * (n + 1) // 2


def _held(c):
    """Elements of the sequences' keys, each sequence its own."""
    return float(sum(s[1] for s in _shape(c)) * c["heads_kv"] * c["d_h"])


def work(case):
    """Bytes and operations one pass cannot do without."""
    c = case
    shape = _shape(c)
    H, hk, D, page = c["heads"], c["heads_kv"], c["d_h"], c["page"]
    rows = sum(s[0] for s in shape)
    o = 4 if c["o_f32"] else 2
    if c["kind"] == "append":
        e = 4 if c["dtype"] == "f32" else 2
        touched = sum((ln - 1) // page - (ln - n) // page + 1 for n, ln, _, _ in shape)
        n = rows * ((H + 2 * hk) * D * e + (H + 2 * hk) * D * 2) + touched * hk * D * 2
        return {"bytes": float(n), "flops": 3.0 * rows * (H + hk) * c["rot"] + rows * hk * D}
    io = rows * H * (D * (2 + o) + 4)
    if c["kind"] == "attn":
        held, seen = 0, set()
        for n, ln, P, g in shape:
            held += ln - (P if g in seen and g >= 0 else 0)
            seen.add(g)
        return {"bytes": float(io + held * hk * D * 4),
                "flops": 4.0 * H * D * sum(_pairs(n, ln) for n, ln, _, _ in shape)}
    byt, flops = float(io), 0.0
    for n, ln, _, _ in shape:
        vis = -(-ln // page)
        sel = min(c["n_sel"], vis)
        byt += vis * hk * D * 2 + min(n * sel, vis) * hk * page * D * 4 + 4 * n * hk * c["n_sel"]
        flops += n * (2.0 * hk * D * vis + 4.0 * H * D * min(sel * page, ln))
    return {"bytes": byt, "flops": flops}


# ---------------------------------------------------------------------------
# Inputs

def _dev(x, dt=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=dt))).to(DEV)


def prepare(case, seed):
    """Inputs from the seed alone: rows, the cache with what earlier calls left in
    it, lengths and tables."""
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    shape = _shape(c)
    H, hk, D, page, B = c["heads"], c["heads_kv"], c["d_h"], c["page"], c["B"]
    table, pages, shared = _tables(c, shape)
    ro = _cum([s[0] for s in shape])
    rows = int(ro[-1])
    s = {"c": c, "n_pages": pages, "rows": rows, "k_max": max(x[0] for x in shape),
         "L_max": max(x[1] for x in shape), "host_offsets": ro,
         "scale": 1.0 / math.sqrt(D), "row_offsets": _dev(ro),
         "lens": _dev([x[1] for x in shape]), "table": _dev(table),
         "prefix_ids": _dev([x[3] for x in shape]) if c["groups"] else None,
         "prefix_lens": _dev([x[2] for x in shape]) if c["groups"] else None,
         "seq": _dev(np.repeat(np.arange(B), np.diff(ro)), np.int64)}
    # keys of a page around a mean of their own, as tokens of one passage are; values
    # around a mean of their head
    K = torch.empty(pages, hk, page, D, dtype=torch.bfloat16, device=DEV)
    V = torch.empty_like(K)
    vm = 0.3 * torch.randn(hk, 1, D, generator=g, device=DEV)
    step = max(1, (1 << 26) // (hk * page * D))
    for i in range(0, pages, step):
        m = min(step, pages - i)
        mu = 0.4 * torch.randn(m, hk, 1, D, generator=g, device=DEV)
        K[i:i + m] = mu + torch.randn(m, hk, page, D, generator=g, device=DEV)
        V[i:i + m] = vm + torch.randn(m, hk, page, D, generator=g, device=DEV)
    for a, b, t in shared:
        K[b, :, :t] = K[a, :, :t]
        V[b, :, :t] = V[a, :, :t]
    s.update(K=K, V=V)
    s["mean"] = None
    if c["kind"] != "attn":
        s["mean"] = torch.empty(pages, hk, D, dtype=torch.bfloat16, device=DEV)
        for i in range(0, pages, step):
            s["mean"][i:i + step] = K[i:i + step].float().mean(2)
    if c["kind"] == "append":
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        if c["packed"]:
            x = torch.randn(rows, (H + 2 * hk) * D, generator=g, device=DEV).to(dt)
            q, k, v = x[:, :H * D], x[:, H * D:(H + hk) * D], x[:, (H + hk) * D:]
        else:
            q, k, v = (torch.randn(rows, h * D, generator=g, device=DEV).to(dt)
                       for h in (H, hk, hk))
        s.update(q=q.view(rows, H, D), k=k.view(rows, hk, D), v=v.view(rows, hk, D))
        s["freq"] = None
        if c["rot"]:
            i = torch.arange(c["rot"] // 2, dtype=torch.float64)
            s["freq"] = torch.pow(10000.0, -2.0 * i / c["rot"]).float().to(DEV)
        s["positions"] = None
        if c["placed"]:
            s["positions"] = torch.sort(torch.randint(0, 9216, (rows,), generator=g, device=DEV)
                                        )[0].to(torch.int32)
    else:
        s["q"] = torch.randn(rows, H, D, generator=g, device=DEV).bfloat16()
    return s


# ---------------------------------------------------------------------------
# One pass

def run(state):
    if own:
        return _run_own(state)
    return {"append": _run_append, "attn": _run_attn, "pages": _run_pages}[state["c"]["kind"]](state)


def _run_own(s):
    c = s["c"]
    if "plan" not in s:                      # what a program keeps from call to call
        from paper_2607_25422_amd import binding as b
        p = b.make_problem(c["dtype"], B=c["B"], d=c["heads"] * c["d_h"], H=c["heads"],
                           d_h=c["d_h"], kept_offsets=s["host_offsets"], sm_scale=s["scale"],
                           o_f32=c["o_f32"])
        p.L_max = s["L_max"]
        cache = b.KvCache(s["K"], s["V"], s["mean"], s["table"])
        rot = None
        if c["kind"] == "append" and s["freq"] is not None:
            rot = b.Rotation(s["freq"], c["style"])
        s["plan"] = b, p, cache, rot
    b, p, cache, rot = s["plan"]
    if c["kind"] == "append":
        q = b.cache_append(p, cache, s["q"], s["k"], s["v"], s["row_offsets"], s["lens"],
                           rotation=rot, positions=s["positions"])
        return q, s["K"], s["V"], s["mean"]
    if c["kind"] == "attn":
        return b.cache_attn(p, cache, s["q"], s["row_offsets"], s["lens"],
                            prefix_ids=s["prefix_ids"], prefix_lens=s["prefix_lens"])
    pages = b.cache_select(p, cache, s["q"], s["row_offsets"], s["lens"], c["n_sel"],
                           n_first=c["n_first"], n_last=c["n_last"])
    O, lse = b.cache_attn_pages(p, cache, s["q"], s["row_offsets"], s["lens"], pages)
    return pages, O, lse


def _rotate(x, ang, style):
    """float32 x [rows, heads, D], its first 2 * ang.shape[1] features rotated by
    the angles (float64)."""
    r = 2 * ang.shape[1]
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    y = x.clone()
    if style == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2] = a * cos - b * sin
        y[..., r // 2:r] = b * cos + a * sin
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2] = a * cos - b * sin
        y[..., 1:r:2] = b * cos + a * sin
    return y


def _token(s):
    """Token of every new row within its sequence."""
    start = s["lens"] - (s["row_offsets"][1:] - s["row_offsets"][:-1])
    row = torch.arange(s["rows"], device=DEV) - s["row_offsets"][s["seq"]]
    return start[s["seq"]].long() + row


def _run_append(s):
    c, page = s["c"], s["c"]["page"]
    tok = _token(s)
    q, k = s["q"].float(), s["k"].float()
    if s["freq"] is not None:
        pos = tok if s["positions"] is None else s["positions"]
        ang = pos.double()[:, None] * s["freq"].double()[None]
        q, k = _rotate(q, ang, c["style"]), _rotate(k, ang, c["style"])
    at = s["table"][s["seq"], tok // page].long()
    s["K"][at, :, tok % page] = k.bfloat16()
    s["V"][at, :, tok % page] = s["v"].bfloat16()
    # mean keys: every page that a row went to, up to the sequence's last token
    held = torch.minimum(s["lens"][s["seq"]].long() - tok // page * page,
                         torch.full_like(tok, page))
    first = torch.cat([torch.ones(1, dtype=torch.bool, device=DEV), at[1:] != at[:-1]])
    pg, held = at[first], held[first]
    there = torch.arange(page, device=DEV)[None] < held[:, None]
    keys = torch.where(there[:, None, :, None], s["K"][pg].float(), torch.zeros((), device=DEV))
    s["mean"][pg] = (keys.sum(2) / held[:, None, None]).bfloat16()
    return q.bfloat16(), s["K"], s["V"], s["mean"]


def _out(c, o, m, l, H, D):
    """Rounded outputs and the logarithm of the sums, [rows, H, D] and [rows, H]."""
    o = torch.where(l > 0, o / l.clamp_min(1e-38), torch.zeros_like(o))
    lse = (m + torch.log(l)).reshape(-1, H)
    return o.reshape(-1, H, D).to(torch.float32 if c["o_f32"] else torch.bfloat16), lse


def _run_attn(s):
    c = s["c"]
    H, hk, D, page, B, n = c["heads"], c["heads_kv"], c["d_h"], c["page"], c["B"], s["k_max"]
    G, L = H // hk, s["L_max"]
    P = -(-L // page)
    tab = s["table"][:, :P].clamp_min(0).long()
    K = s["K"][tab].permute(0, 2, 4, 1, 3).reshape(B, hk, D, P * page).float()
    V = s["V"][tab].permute(0, 2, 1, 3, 4).reshape(B, hk, P * page, D).float()
    row = torch.arange(s["rows"], device=DEV) - s["row_offsets"][s["seq"]]
    q = torch.zeros(B, hk, G, n, D, device=DEV)
    q[s["seq"], :, :, row] = s["q"].float().view(-1, hk, G, D)
    tok = torch.full((B, n), -1, dtype=torch.int64, device=DEV)
    tok[s["seq"], row] = _token(s)
    z = (q.view(B, hk, G * n, D) @ K).view(B, hk, G, n, P * page)
    z *= s["scale"]
    z.masked_fill_((torch.arange(P * page, device=DEV) > tok[..., None])[:, None, None],
                   float("-inf"))
    m = z.amax(-1, keepdim=True).clamp_min(-3e38)
    z -= m
    p = z.exp_()
    l = p.sum(-1, keepdim=True)
    o = (p.view(B, hk, G * n, P * page) @ V).view(B, hk, G, n, D)
    o, m, l = (x[s["seq"], :, :, row] for x in (o, m, l))
    return _out(c, o, m, l, H, D)


def _run_pages(s):
    c = s["c"]
    H, hk, D, page, B, n = c["heads"], c["heads_kv"], c["d_h"], c["page"], c["B"], s["k_max"]
    G, L, M = H // hk, s["L_max"], s["rows"]
    P = -(-L // page)
    tok = _token(s)
    tab = s["table"][:, :P].clamp_min(0).long()
    # scores in 64 bits: a cut between neighbouring values
    row = torch.arange(M, device=DEV) - s["row_offsets"][s["seq"]]
    q = torch.zeros(B, hk, n, D, dtype=torch.float64, device=DEV)
    q[s["seq"], :, row] = s["q"].double().view(M, hk, G, D).sum(2)
    z = (q @ s["mean"][tab].permute(0, 2, 3, 1).double().contiguous())[s["seq"], :, row]
    j = torch.arange(P, device=DEV)[None]
    last = (tok // page)[:, None]
    always = (j < c["n_first"]) | (j > last - c["n_last"])
    z = z.masked_fill(always[:, None], float("inf")).masked_fill((j > last)[:, None], float("-inf"))
    order = torch.sort(z, dim=-1, descending=True, stable=True).indices[..., :c["n_sel"]]
    order = torch.where(order <= last[:, None], order, torch.full_like(order, P))
    order = torch.sort(order, dim=-1).values
    sel = torch.full((M, hk, c["n_sel"]), -1, dtype=torch.int32, device=DEV)
    sel[..., :order.shape[-1]] = torch.where(order < P, order, torch.full_like(order, -1))
    # attention over them
    at = tab[s["seq"][:, None, None], sel.clamp_min(0).long()]            # rows, hk, n_sel
    heads = torch.arange(hk, device=DEV)[None, :, None]
    t = sel.long()[..., None] * page + torch.arange(page, device=DEV)
    seen = ((sel >= 0)[..., None] & (t <= tok[:, None, None, None])).view(M, hk, 1, -1)
    k = s["K"][at, heads].view(M, hk, -1, D).float()
    z = (s["q"].float().view(M, hk, G, D) @ k.transpose(2, 3).contiguous()) * s["scale"]
    z = z.masked_fill(~seen, float("-inf"))
    m = z.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(z - m)
    l = p.sum(-1, keepdim=True)
    o = p @ s["V"][at, heads].view(M, hk, -1, D).float()
    return (sel, *_out(c, o, m, l, H, D))


# ---------------------------------------------------------------------------
# The operators' definitions in 64 bits, a sequence at a time

def exact(case, seed):
    c = case
    shape = _shape(c)
    if work(c)["flops"] > 4e12 or (c["kind"] == "pages" and
                                   sum(x[0] for x in shape) * c["heads_kv"] > 10000):
        return None
    s = prepare(c, seed)
    H, hk, D, page = c["heads"], c["heads_kv"], c["d_h"], c["page"]
    table = s["table"].cpu().numpy()
    O = torch.zeros(s["rows"], H, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["rows"], H, dtype=torch.float64, device=DEV)
    sel = torch.full((s["rows"], hk, max(1, c["n_sel"])), -1, dtype=torch.int32, device=DEV)
    if c["kind"] == "append":
        K, V, mean = s["K"].double(), s["V"].double(), s["mean"].double()
    r0 = 0
    for b, (n, ln, _, _) in enumerate(shape):
        own_pages = torch.from_numpy(table[b, :-(-ln // page)].astype(np.int64)).to(DEV)
        rows = slice(r0, r0 + n)
        if c["kind"] == "append":
            q, k, v = (s[x][rows].double() for x in "qkv")
            pos = (torch.arange(ln - n, ln, device=DEV) if s["positions"] is None
                   else s["positions"][rows])
            for h in range(0, c["rot"] // 2):
                i, j = (h, h + c["rot"] // 2) if c["style"] == "halves" else (2 * h, 2 * h + 1)
                turn = torch.polar(torch.ones(n, dtype=torch.float64, device=DEV),
                                   pos.double() * float(s["freq"][h]))[:, None]
                for x in (q, k):
                    w = torch.complex(x[..., i], x[..., j]) * turn
                    x[..., i], x[..., j] = w.real, w.imag
            O[rows] = q
            for t0 in range((ln - n) // page * page, ln, page):
                at, a, e = own_pages[t0 // page], max(t0, ln - n), min(t0 + page, ln)
                K[at, :, a - t0:e - t0] = k[a - (ln - n):e - (ln - n)].transpose(0, 1)
                V[at, :, a - t0:e - t0] = v[a - (ln - n):e - (ln - n)].transpose(0, 1)
                # (the mean of the keys as the cache holds them)
                mean[at] = K[at, :, :e - t0].bfloat16().double().mean(1)
        elif c["kind"] == "attn":
            k = s["K"][own_pages].transpose(1, 2).reshape(-1, hk, D)[:ln].double()
            v = s["V"][own_pages].transpose(1, 2).reshape(-1, hk, D)[:ln].double()
            for h in range(H):
                e = s["q"][rows, h].double() @ k[:, h * hk // H].t().contiguous() * s["scale"]
                e += torch.full_like(e, float("-inf")).triu(ln - n + 1)
                lse[rows, h] = torch.logsumexp(e, 1)
                O[rows, h] = torch.softmax(e, 1) @ v[:, h * hk // H]
        else:
            means = s["mean"][own_pages].double()
            for i in range(n):
                t, qi = ln - n + i, s["q"][r0 + i].double().view(hk, H // hk, D)
                vis = t // page + 1
                for h in range(hk):
                    score = (means[:vis, h] * qi[h].sum(0)).sum(1)
                    score[:c["n_first"]] = float("inf")
                    score[max(0, vis - c["n_last"]):] = float("inf")
                    take = torch.sort(torch.sort(score, descending=True,
                                                 stable=True)[1][:c["n_sel"]])[0]
                    sel[r0 + i, h, :len(take)] = take.to(torch.int32)
                    k, v = (s[x][own_pages[take], h].reshape(-1, D).double() for x in "KV")
                    tok = (take[:, None] * page + torch.arange(page, device=DEV)).flatten()
                    e = (qi[h] @ k.t().contiguous() * s["scale"])[:, tok <= t]
                    heads = slice(h * (H // hk), (h + 1) * (H // hk))
                    lse[r0 + i, heads] = torch.logsumexp(e, 1)
                    O[r0 + i, heads] = torch.softmax(e, 1) @ v[tok <= t]
        r0 += n
    if c["kind"] == "append":
        return O, K, V, mean
    return (O, lse) if c["kind"] == "attn" else (sel, O, lse)
