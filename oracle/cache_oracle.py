"""Plain float64 definitions of the paged cache's operators (numpy, one sequence at
a time).  A cache is (k, v, mean, table): k, v [pages, heads_kv, page, d_h], mean
[pages, heads_kv, d_h], table [B, pages_max]; arrays of float64 values.  Sequence b has
the rows row_offsets[b] .. row_offsets[b + 1] - 1, the last of its lens[b] tokens.
"""
from __future__ import annotations

import numpy as np


def rotate(x, pos, freq, style):
    """x [rows, heads, d_h], the first 2 * len(freq) features rotated by pos * freq."""
    ang = np.asarray(pos, dtype=np.float64)[:, None] * np.asarray(freq, dtype=np.float64)[None]
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    r, y = 2 * len(freq), x.copy()
    i = slice(0, r // 2) if style == "halves" else slice(0, r, 2)
    j = slice(r // 2, r) if style == "halves" else slice(1, r, 2)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def tokens(row_offsets, lens, b):
    """Tokens of sequence b's rows."""
    n = int(row_offsets[b + 1] - row_offsets[b])
    return np.arange(int(lens[b]) - n, int(lens[b]))


def page_slots(table, page, b, tok):
    return np.asarray(table)[b, np.asarray(tok) // page], np.asarray(tok) % page


def gather(x, table, page, b, n):
    """The first n tokens of sequence b, [n, heads_kv, d_h] (0 where the page is
    missing), and whether each is there."""
    at, slot = page_slots(table, page, b, np.arange(n))
    there = (at >= 0) & (at < x.shape[0])
    return np.where(there[:, None, None], x[np.where(there, at, 0), :, slot], 0.0), there


def softmax_rows(q, k, v, seen, scale):
    """One head: q [rows, d], k, v [tokens, d], seen [rows, tokens] -> (O, lse, sum of
    weights times |v|)."""
    e = np.where(seen, q @ np.where(seen.any(0)[:, None], k, 0.0).T * scale, -np.inf)
    m = np.max(e, axis=1, initial=-np.inf)
    p = np.exp(e - np.where(np.isfinite(m), m, 0.0)[:, None])
    l = p.sum(1)
    p = p / np.where(l > 0, l, 1.0)[:, None]
    vz = np.where(seen.any(0)[:, None], v, 0.0)
    with np.errstate(divide="ignore"):
        return p @ vz, np.where(l > 0, m + np.log(np.where(l > 0, l, 1.0)), -np.inf), p @ np.abs(vz)


def attention(q, k, v, table, row_offsets, lens, scale, listed=None):
    """q [rows, H, d_h] -> (O, lse, weights times |v|) of every row; listed
    [rows, heads_kv, n_sel]: the pages that count, each as often as it is named."""
    rows, H, D = q.shape
    hk, page = k.shape[1], k.shape[2]
    O, A, lse = np.zeros((rows, H, D)), np.zeros((rows, H, D)), np.full((rows, H), -np.inf)
    for b in range(len(lens)):
        r0 = int(row_offsets[b])
        tok = tokens(row_offsets, lens, b)
        K, there = gather(k, table, page, b, int(lens[b]))
        V, _ = gather(v, table, page, b, int(lens[b]))
        for h in range(H):
            g = h * hk // H
            if listed is None:
                seen = there[None] & (np.arange(int(lens[b]))[None] <= tok[:, None])
                for i in range(len(tok)):            # (what a row does not see is not read)
                    s = seen[i]
                    o = softmax_rows(q[r0 + i:r0 + i + 1, h], K[s, g], V[s, g],
                                     np.ones((1, s.sum()), bool), scale)
                    O[r0 + i, h], lse[r0 + i, h], A[r0 + i, h] = o[0][0], o[1][0], o[2][0]
                continue
            for i, t in enumerate(tok):
                at = [j * page + s for j in listed[r0 + i, g] if 0 <= j <= t // page and t >= 0
                      for s in range(page) if j * page + s <= t and there[j * page + s]]
                o = softmax_rows(q[r0 + i:r0 + i + 1, h], K[at, g], V[at, g],
                                 np.ones((1, len(at)), bool), scale)
                O[r0 + i, h], lse[r0 + i, h], A[r0 + i, h] = o[0][0], o[1][0], o[2][0]
    return O, lse, A


def select(q, mean, table, page, row_offsets, lens, n_sel, n_first, n_last):
    """Pages of every row and key head, [rows, heads_kv, n_sel]."""
    rows, H, D = q.shape
    hk = mean.shape[1]
    out = np.full((rows, hk, n_sel), -1, dtype=np.int32)
    qs = q.reshape(rows, hk, H // hk, D).sum(2)
    for b in range(len(lens)):
        for i, t in enumerate(tokens(row_offsets, lens, b)):
            r, vis = int(row_offsets[b]) + i, (t // page + 1 if t >= 0 else 0)
            at = np.asarray(table)[b, :vis]
            there = (at >= 0) & (at < mean.shape[0])
            for h in range(hk):
                z = np.where(there, mean[np.where(there, at, 0), h] @ qs[r, h], 0.0)
                j = np.arange(vis)
                always = (j < n_first) | (j >= vis - n_last)
                order = sorted(range(vis), key=lambda x: (not always[x], -z[x], x))[:n_sel]
                out[r, h, :len(order)] = sorted(order)
    return out
