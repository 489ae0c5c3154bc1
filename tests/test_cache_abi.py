"""Refusals of the paged cache's calls, on the host (every call here fails its checks
before anything is enqueued), and its oracle in closed forms."""
import ctypes

import numpy as np
import pytest

from oracle import cache_oracle as co

FAKE = 1 << 40   # never dereferenced


@pytest.fixture(scope="module")
def b():
    from paper_2607_25422_amd import binding
    return binding


def problem(b, dtype="bf16", L_max=200, **kw):
    base = dict(B=2, d=1024, H=16, d_h=64, kept_offsets=[0, 3, 5], sm_scale=0.125)
    base.update(kw)
    p = b.make_problem(dtype, **base)
    p.L_max = L_max
    return p


def cache(b, **kw):
    a = dict(heads_kv=4, page_tokens=64, pages_max=8, reserved=0, n_pages=20, k=FAKE, v=FAKE,
             mean=FAKE, page_table=FAKE)
    a.update(kw)
    return b.SkipKvCache(*a.values())


BAD_CACHES = [dict(heads_kv=0), dict(heads_kv=5), dict(pages_max=0), dict(pages_max=3),
              dict(reserved=1), dict(n_pages=0), dict(n_pages=1 << 31), dict(k=None), dict(v=None),
              dict(page_table=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(mean=FAKE + 4)]
ODD_CACHES = [dict(page_tokens=16), dict(page_tokens=0), dict(page_tokens=96),
              dict(page_tokens=512)]


def call(b, fn, p, c, **kw):
    ref = lambda x: None if x is None else ctypes.byref(x)
    a = dict(rot=None, q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, ro=FAKE, lens=FAKE,
             pos=None, qo=FAKE, ids=None, pls=None, pages=FAKE, n_sel=4, n_first=1, n_last=1,
             O=FAKE, lse=None, ws=FAKE, nb=1 << 40)
    a.update(kw)
    g = lambda *names: [a[n] for n in names]
    if fn == "append":
        return b.LIB.skip_cache_append(ref(p), ref(c), ref(a["rot"]),
                                       *g("q", "qs", "k", "ks", "v", "vs", "ro", "lens", "pos",
                                          "qo"), None)
    if fn == "attn":
        return b.LIB.skip_cache_attn(ref(p), ref(c), *g("q", "ro", "lens", "ids", "pls", "O", "lse",
                                                        "ws", "nb"), None)
    if fn == "select":
        return b.LIB.skip_cache_select(ref(p), ref(c), *g("q", "ro", "lens", "n_sel", "n_first",
                                                          "n_last", "pages", "ws", "nb"), None)
    return b.LIB.skip_cache_attn_pages(ref(p), ref(c), *g("q", "ro", "lens", "pages", "n_sel", "O",
                                                          "lse", "ws", "nb"), None)


ALL = ("append", "attn", "select", "pages")


def test_structs(b):
    assert ctypes.sizeof(b.SkipKvCache) == 56 and b.SkipKvCache.k.offset == 24
    assert ctypes.sizeof(b.SkipRotation) == 16


@pytest.mark.parametrize("fn", ALL)
def test_cache_and_problem(b, fn):
    inv, uns = b.SKIP_ERR_INVALID_ARG, b.SKIP_ERR_UNSUPPORTED
    assert call(b, fn, None, cache(b)) == inv and call(b, fn, problem(b), None) == inv
    for kw in BAD_CACHES:
        assert call(b, fn, problem(b), cache(b, **kw)) == inv, kw
    for kw in ODD_CACHES:
        assert call(b, fn, problem(b), cache(b, **kw)) == uns, kw
    for kw in (dict(ro=None), dict(lens=None), dict(q=FAKE + 8)):
        assert call(b, fn, problem(b), cache(b), **kw) == inv, kw
    assert call(b, fn, problem(b, d=512), cache(b)) == inv                 # H * d_h != d
    assert call(b, fn, problem(b, H=32, d_h=32), cache(b)) == uns
    assert call(b, fn, problem(b, H=64, d=4096), cache(b, heads_kv=1)) == uns   # 64 to a key head
    assert call(b, fn, problem(b, L_max=513), cache(b)) == inv             # past the page table
    assert call(b, fn, problem(b, L_max=-1), cache(b)) == inv
    assert call(b, fn, problem(b, L_max=(1 << 30) + 1), cache(b, pages_max=1 << 30)) == uns
    assert call(b, fn, problem(b, sm_scale=float("nan")), cache(b)) == inv
    # no rows: nothing to do
    none = problem(b, kept_offsets=[0, 0, 0])
    assert call(b, fn, none, cache(b), q=None, k=None, v=None, qo=None, pages=None, O=None,
                ws=None, nb=0) == b.SKIP_OK


def test_append(b):
    inv, uns = b.SKIP_ERR_INVALID_ARG, b.SKIP_ERR_UNSUPPORTED
    p, c = problem(b), cache(b)
    for kw in (dict(k=None), dict(v=None), dict(qo=None), dict(k=FAKE + 2), dict(v=FAKE + 8),
               dict(qo=FAKE + 4), dict(ks=248), dict(vs=0), dict(qs=1016), dict(ks=260),
               dict(vs=-256), dict(qs=1028)):
        assert call(b, "append", p, c, **kw) == inv, kw
    for rot, st in (((None, 64, 0), inv), ((FAKE, 64, 2), inv), ((FAKE, 8, 0), inv),
                    ((FAKE, 80, 0), inv), ((FAKE, 24, 0), uns)):
        assert call(b, "append", p, c, rot=b.SkipRotation(*rot)) == st, rot


def test_attention(b):
    inv, uns = b.SKIP_ERR_INVALID_ARG, b.SKIP_ERR_UNSUPPORTED
    c = cache(b, pages_max=100)
    p = problem(b, L_max=6000)
    for fn in ("attn", "pages", "select"):
        assert call(b, fn, problem(b, dtype="f32"), c) == uns
        assert call(b, fn, p, c, q=None) == inv
        assert call(b, fn, p, c, ws=FAKE + 8) == inv
    for fn in ("attn", "pages"):
        assert call(b, fn, p, c, O=None) == inv and call(b, fn, p, c, O=FAKE + 4) == inv
    for kw in (dict(ids=FAKE), dict(pls=FAKE)):
        assert call(b, "attn", p, c, **kw) == inv, kw
    long = problem(b, L_max=64 * 2000)                       # (scores in a launch of their own)
    wide = cache(b, pages_max=2000)
    for fn, n_sel, pre, p, c in (("attn", 0, 0, p, c), ("attn", 0, 1, p, c),
                                 ("pages", 90, 0, p, c), ("select", 9, 0, long, wide)):
        need = ctypes.c_size_t(0)
        assert b.LIB.skip_workspace_bytes_cache(ctypes.byref(p), ctypes.byref(c), n_sel, pre,
                                                ctypes.byref(need)) == b.SKIP_OK
        assert need.value > 0
        kw = dict(n_sel=max(n_sel, 1))
        if pre:
            kw.update(ids=FAKE, pls=FAKE)
        if fn != "select":
            assert call(b, fn, p, c, nb=need.value - 1, **kw) == b.SKIP_ERR_WORKSPACE
        assert call(b, fn, p, c, nb=7, **kw) == b.SKIP_ERR_WORKSPACE
        assert call(b, fn, p, c, ws=None, **kw) == inv
    p, c = problem(b, L_max=6000), cache(b, pages_max=100)
    # up to 512 tokens a sequence: none, whatever the rows
    for pre in (0, 1):
        for H, d_h, n in ((16, 64, 1), (16, 64, 9), (32, 128, 500), (64, 64, 2000), (12, 64, 3)):
            short = problem(b, B=70, H=H, d=H * d_h, d_h=d_h, L_max=512,
                            kept_offsets=[0] + list(range(n, 70 + n)))
            assert b.LIB.skip_workspace_bytes_cache(ctypes.byref(short), ctypes.byref(c), 0, pre,
                                                    ctypes.byref(need)) == b.SKIP_OK
            assert need.value == 0
    # listed pages of up to 512 tokens, selection of up to 1024 pages: none
    for page in (32, 64, 128, 256):
        wide = cache(b, page_tokens=page, pages_max=1024)
        for n in (1, 40, 3000):
            for L in (5, 1024 * page):
                short = problem(b, kept_offsets=[0, 1, n + 1], L_max=L)
                assert b.LIB.skip_workspace_bytes_cache(
                    ctypes.byref(short), ctypes.byref(wide), 512 // page, 0,
                    ctypes.byref(need)) == b.SKIP_OK
                assert need.value == 0
    p, c = problem(b, L_max=6000), cache(b, pages_max=100)
    assert b.LIB.skip_workspace_bytes_cache(ctypes.byref(p), ctypes.byref(c), 0, 0, None) == inv
    assert b.LIB.skip_workspace_bytes_cache(ctypes.byref(p), ctypes.byref(c), -1, 0,
                                            ctypes.byref(need)) == inv
    # more than 2^30 blocks of work
    wide = problem(b, B=4096, kept_offsets=list(range(4097)), L_max=1 << 30)
    assert call(b, "attn", wide, cache(b, pages_max=1 << 30)) == uns


def test_scales_past_float32(b):
    """The scale enters in base 2: one whose product with log2 e is infinite is refused by
    the calls that use it."""
    c = cache(b)
    for scale in (2.5e38, -3.4e38):
        p = problem(b, sm_scale=scale)
        for fn in ("attn", "pages"):
            assert call(b, fn, p, c) == b.SKIP_ERR_INVALID_ARG, (fn, scale)


def test_workspace_where_only_one_of_the_two_calls_is_possible(b):
    """Rows and pages past the selection's limits: the attention's need.  More tiles of
    listed pages than are counted: the selection's.  Neither: refused."""
    def need(p, c, n_sel):
        n = ctypes.c_size_t(77)
        return b.LIB.skip_workspace_bytes_cache(ctypes.byref(p), ctypes.byref(c), n_sel, 0,
                                                ctypes.byref(n)), n.value
    ok, uns = b.SKIP_OK, b.SKIP_ERR_UNSUPPORTED
    # 512 items and more, taken whole: none
    many = problem(b, B=1, kept_offsets=[0, 70000], L_max=6400)
    assert need(many, cache(b, pages_max=100), 32) == (ok, 0)
    # 16385 pages a sequence: parts of 512 runs of 16 rows and 66 floats, and 10 counts
    long = problem(b, L_max=64 * 16384 + 1)
    wide = cache(b, pages_max=16385)
    assert need(long, wide, 32) == (ok, 2 * 512 * 16 * 66 * 4 + 256)
    assert call(b, "pages", long, wide, n_sel=32, nb=7) == b.SKIP_ERR_WORKSPACE
    assert call(b, "select", long, wide, n_sel=32) == uns
    assert call(b, "select", many, cache(b, pages_max=100), n_sel=32) == uns
    # 2^17 rows and key heads times 8200 tiles; 3000 pages, scores in LDS
    deep = problem(b, B=1, H=16, kept_offsets=[0, 1 << 13], L_max=256 * 3000)
    c = cache(b, heads_kv=16, page_tokens=256, pages_max=3000)
    assert call(b, "pages", deep, c, n_sel=1024) == uns and need(deep, c, 1024) == (ok, 0)
    far = problem(b, B=1, H=16, kept_offsets=[0, 1 << 13], L_max=256 * 16385)
    assert need(far, cache(b, heads_kv=16, page_tokens=256, pages_max=16385), 1024)[0] == uns


@pytest.mark.parametrize("H,hk,d_h", [(96, 8, 128), (129, 129, 64), (2048, 64, 128),
                                      (65535, 65535, 128)])
def test_wide_rows(b, H, hk, d_h):
    """Rows wider than the routes take: no limit of the cache's calls but its own ones."""
    p = problem(b, H=H, d=H * d_h, d_h=d_h, L_max=500)
    c = cache(b, heads_kv=hk)
    need = ctypes.c_size_t(0)
    for n_sel in (0, 4):
        assert b.LIB.skip_workspace_bytes_cache(ctypes.byref(p), ctypes.byref(c), n_sel, 0,
                                                ctypes.byref(need)) == b.SKIP_OK
    none = problem(b, H=H, d=H * d_h, d_h=d_h, kept_offsets=[0, 0, 0])
    for fn in ALL:
        assert call(b, fn, none, c) == b.SKIP_OK
        assert call(b, fn, p, c, q=None, k=None, pages=None) == b.SKIP_ERR_INVALID_ARG
    assert call(b, "append", p, c, qs=H * d_h - 8, ks=hk * d_h, vs=hk * d_h) == b.SKIP_ERR_INVALID_ARG


def test_more_than_a_launch_holds(b):
    uns = b.SKIP_ERR_UNSUPPORTED

    def big(B, rows, k_max, **kw):
        p = problem(b, **kw)
        p.B, p.total_kept, p.k_max = B, rows, k_max
        return p
    one = cache(b, heads_kv=1)
    kw = dict(H=1, d=64, d_h=64)
    strides = dict(qs=64, ks=64, vs=64)
    for B, rows, k_max in ((1 << 24, 1 << 24, 1), (1 << 23, 1 << 30, 1 << 8)):
        p = big(B, rows, k_max, L_max=500, **kw)
        assert call(b, "append", p, one, **strides) == uns, (B, rows)
        assert call(b, "attn", p, one) == uns, (B, rows)
        assert call(b, "pages", p, one) == uns, (B, rows)
    many = cache(b, heads_kv=65536)
    p = problem(b, H=65536, d=65536 * 64, d_h=64)
    for fn in ALL:
        assert call(b, fn, p, many, qs=p.d, ks=p.d, vs=p.d) == uns, fn
    wide = cache(b, heads_kv=16384)
    p = problem(b, H=16384, d=16384 * 64, d_h=64, B=1, kept_offsets=[0, 4096])
    assert call(b, "select", p, wide) == uns
    # the tiles of all blocks just past what is counted
    p = big(1, 1 << 20, 1 << 20, L_max=32 * 16384, **kw)
    assert call(b, "attn", p, cache(b, heads_kv=1, pages_max=8192)) == uns


def test_selection(b):
    inv, uns = b.SKIP_ERR_INVALID_ARG, b.SKIP_ERR_UNSUPPORTED
    p, c = problem(b), cache(b)
    for kw in (dict(n_sel=0), dict(n_sel=-1), dict(pages=None)):
        assert call(b, "select", p, c, **kw) == inv and call(b, "pages", p, c, **kw) == inv, kw
    for fn in ("select", "pages"):
        assert call(b, fn, p, c, n_sel=1025) == uns
    for kw in (dict(n_first=-1), dict(n_last=0), dict(n_first=4), dict(n_last=4),
               dict(n_first=(1 << 31) - 1, n_last=(1 << 31) - 1)):
        assert call(b, "select", p, c, **kw) == inv, kw
    assert call(b, "select", p, cache(b, mean=None)) == inv
    assert call(b, "select", problem(b, L_max=64 * 16384 + 1), cache(b, pages_max=20000)) == uns
    assert call(b, "select", problem(b, B=1, kept_offsets=[0, 65536]), c) == uns


def test_binding_checks(b):
    """Shapes are compared before any pointer goes to the library."""
    import torch
    p = problem(b)
    kv = torch.empty(20, 4, 64, 64, dtype=torch.bfloat16)
    t = torch.zeros(2, 8, dtype=torch.int32)
    build = lambda *a: b._cache_struct(p, b.KvCache(*a), 0)
    with pytest.raises(ValueError, match="page_tokens"):
        build(kv, kv[:3], None, t)
    with pytest.raises(ValueError, match="pages_max"):
        build(kv, kv, None, t[0])
    with pytest.raises(ValueError, match="device"):
        build(kv, kv, None, t)
    # known arrays: the problem's sizes and the device are compared at every call
    c = b.KvCache(kv, kv, None, t)
    at = (kv.data_ptr(), kv.data_ptr(), None, t.data_ptr())
    c.__dict__["_struct"] = known = (b.SkipKvCache(4, 64, 8, 0, 20, *at), 64, 2, 0, at,
                                       (kv.numel(), t.numel()))
    assert b._cache_struct(p, c, 0).k == kv.data_ptr()
    with pytest.raises(ValueError, match="device 0"):
        b._cache_struct(p, c, 1)
    with pytest.raises(ValueError, match="128"):
        b._cache_struct(problem(b, d=2048, d_h=128), c, 0)
    with pytest.raises(ValueError, match="3 rows"):
        b._cache_struct(problem(b, B=3, kept_offsets=[0, 1, 2, 3]), c, 0)
    # arrays that are set anew are looked at anew
    c.page_table = t[0]
    with pytest.raises(ValueError, match="pages_max"):
        b._cache_struct(p, c, 0)
    # and so are those that were given other memory in place
    c = b.KvCache(kv, kv, None, t.clone())
    c.__dict__["_struct"] = known[:4] + (at[:3] + (c.page_table.data_ptr(),), known[5])
    assert b._cache_struct(p, c, 0) is known[0]
    c.page_table.resize_(1, 8)
    with pytest.raises(ValueError, match="device"):          # (looked at, and not on one)
        b._cache_struct(p, c, 0)
    c.page_table.resize_(2, 8)
    assert b._cache_struct(p, c, 0) is known[0]
    c.page_table.set_(torch.zeros(16, dtype=torch.int32))
    with pytest.raises(ValueError, match="pages_max"):
        b._cache_struct(p, c, 0)


def test_binding_looks_at_a_changed_rotation(b):
    import torch
    r = b.Rotation(torch.ones(16))
    key = (r.freq.data_ptr(), 16, "halves", 0)
    r.__dict__["_struct"] = known = (key, b.SkipRotation(r.freq.data_ptr(), 32, 0))
    assert b._rotation_struct(r, 0) is known[1]
    r.freq.resize_(8)
    with pytest.raises(ValueError, match="device"):          # (looked at, and not on one)
        b._rotation_struct(r, 0)
    r.freq.resize_(16)
    assert b._rotation_struct(r, 0) is known[1]
    for change in (lambda: setattr(r, "style", "pairs"), lambda: setattr(r, "freq", torch.ones(24))):
        r.__dict__["_struct"] = known
        change()
        with pytest.raises(ValueError, match="device"):
            b._rotation_struct(r, 0)


def test_binding_looks_at_arrays_changed_in_place(b):
    """What keeps an array's address and may keep its count of elements: other sizes, an
    exchange of dimensions, another type."""
    import torch
    p = problem(b)

    def known(mean=False, B=2, pages_max=8):
        k = torch.empty(20, 4, 64, 64, dtype=torch.bfloat16)
        v, t = torch.empty_like(k), torch.zeros(B, pages_max, dtype=torch.int32)
        m = torch.empty(20, 4, 64, dtype=torch.bfloat16) if mean else None
        c = b.KvCache(k, v, m, t)
        at = (k.data_ptr(), v.data_ptr(), m.data_ptr() if mean else None, t.data_ptr())
        s = (b.SkipKvCache(4, 64, pages_max, 0, 20, *at), 64, B, 0, at, (k.numel(), t.numel()))
        c.__dict__["_struct"] = s
        assert b._cache_struct(p, c, 0) is s[0]
        return c

    def set_data(x, dtype):
        x.data = x.view(dtype)
    for change in (lambda c: c.page_table.resize_(4, 4), lambda c: c.k.resize_(20, 8, 32, 64),
                   lambda c: c.k.resize_(40, 4, 32, 64), lambda c: c.v.resize_(10, 4, 64, 64),
                   lambda c: c.k.transpose_(2, 3), lambda c: c.v.transpose_(2, 3),
                   lambda c: set_data(c.k, torch.float16), lambda c: set_data(c.v, torch.int16),
                   lambda c: set_data(c.page_table, torch.float32)):
        c = known()
        change(c)
        with pytest.raises(ValueError):                      # (looked at, and not on a device)
            b._cache_struct(p, c, 0)
    c = known(B=8)
    c.page_table.t_()
    with pytest.raises(ValueError):
        b._cache_struct(p, c, 0)
    for change in (lambda m: m.resize_(10, 4, 64), lambda m: m.resize_(0),
                   lambda m: m.transpose_(0, 1), lambda m: set_data(m, torch.float16)):
        c = known(mean=True)
        change(c.mean)
        with pytest.raises(ValueError):
            b._cache_struct(p, c, 0)
    r = b.Rotation(torch.ones(16))
    r.__dict__["_struct"] = ((r.freq.data_ptr(), 16, "halves", 0),
                             b.SkipRotation(r.freq.data_ptr(), 32, 0))
    b._rotation_struct(r, 0)
    r.freq.data = r.freq.view(torch.int32)
    with pytest.raises(ValueError):
        b._rotation_struct(r, 0)
    r.freq.data = torch.as_strided(torch.ones(32), (16,), (2,))
    with pytest.raises(ValueError):
        b._rotation_struct(r, 0)


def test_caches_and_rotations_are_copied_and_pickled(b):
    """The kept description, whose pointers are this process's, stays behind."""
    import copy
    import pickle
    import torch
    c = b.KvCache(torch.ones(2, 1, 32, 64), torch.zeros(2, 1, 32, 64), None, torch.zeros(1, 2))
    r = b.Rotation(torch.ones(16), "pairs")
    c.__dict__["_struct"] = (b.SkipKvCache(1, 32, 2, 0, 2, 4096, 4096, None, 4096),)
    r.__dict__["_struct"] = (None, b.SkipRotation(4096, 32, 1))
    for x in (c, r):
        for y in (copy.copy(x), copy.deepcopy(x), pickle.loads(pickle.dumps(x))):
            assert "_struct" not in y.__dict__ and type(y) is type(x)
            for name in ("k", "v", "mean", "page_table") if x is c else ("freq",):
                a, z = getattr(x, name), getattr(y, name)
                assert (a is z is None) or torch.equal(a, z)
        assert "_struct" in x.__dict__
    assert copy.copy(r).style == "pairs" and copy.copy(c).k is c.k


# ---------------------------------------------------------------------------
# The oracle

def test_oracle_rotation():
    x = np.zeros((2, 1, 6))
    x[:, 0] = [1, 2, 3, 4, 5, 6]
    half_turn = co.rotate(x, [1, 0], [np.pi, np.pi], "halves")
    assert np.allclose(half_turn[0, 0], [-1, -2, -3, -4, 5, 6]) and (half_turn[1] == x[1]).all()
    quarter = co.rotate(x, [2, 0], [np.pi / 4, 0.0], "pairs")
    assert np.allclose(quarter[0, 0], [-2, 1, 3, 4, 5, 6])
    # a product of two rotated rows depends on the distance of their positions alone
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 8))
    for style in ("halves", "pairs"):
        dots = [float((co.rotate(q, [a], [0.3, 0.01], style) *
                       co.rotate(k, [a + 5], [0.3, 0.01], style)).sum()) for a in (0, 17, 90000)]
        assert np.allclose(dots, dots[0])


def test_oracle_attention():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 3, 1, 4, 8))
    table, ro, lens = np.array([[2, 0], [1, -1]]), [0, 2, 3], [6, 1]
    q = rng.standard_normal((3, 2, 8))
    O, lse, _ = co.attention(q, k, v, table, ro, lens, 0.0)
    toks = np.concatenate([v[2, 0], v[0, 0]])
    assert np.allclose(O[0], toks[:5].mean(0)) and np.allclose(O[1], toks[:6].mean(0))
    assert np.allclose(O[2], v[1, 0, 0]) and np.allclose(lse, np.log([[5], [6], [1]]))
    listed = np.full((3, 1, 2), -1)
    listed[1, 0] = [1, 1]
    O, lse, _ = co.attention(q, k, v, table, ro, lens, 0.0, listed)
    assert np.allclose(O[1], toks[4:6].mean(0)) and np.allclose(lse[1], np.log(4))
    assert (O[0] == 0).all() and (lse[0] == -np.inf).all()


def test_oracle_selection():
    mean = np.array([3., 1., 2., 2., 5.])[:, None, None] * np.ones((5, 1, 4))
    q = np.ones((1, 2, 4))
    pick = lambda **kw: co.select(q, mean, np.array([[0, 1, 2, 3, 4]]), 4, [0, 1], [20],
                                  **kw)[0, 0].tolist()
    assert pick(n_sel=3, n_first=0, n_last=1) == [0, 2, 4]            # a tie: the lower page
    assert pick(n_sel=3, n_first=2, n_last=1) == [0, 1, 4]
    assert pick(n_sel=7, n_first=1, n_last=1) == [0, 1, 2, 3, 4, -1, -1]
