"""Refusals of the layer calls, on the host."""
import ctypes

import pytest

FAKE = 1 << 40   # never dereferenced


@pytest.fixture(scope="module")
def b():
    from paper_2607_25422_amd import binding
    return binding


def problem(b, **kw):
    base = dict(B=2, N=576, d=1024, kept_offsets=[0, 96, 192])
    dtype = kw.pop("dtype", "bf16")
    base.update(kw)
    return b.make_problem(dtype, **base)


def test_sizes(b):
    assert b.packed_bytes_dense(problem(b), 8) == 256 * 1024 * 2
    assert b.packed_bytes_dense(problem(b), 264) == 512 * 1024 * 2
    assert b.packed_bytes_dense(problem(b, d=16384), 256) == 256 * 16384 * 2
    assert b.workspace_bytes_dense(problem(b, kept_offsets=[0, 0, 0]), 256) == 0
    n = b.workspace_bytes_dense(problem(b, d=16384, kept_offsets=[0, 1, 2]), 256)
    assert n % (2 * 256 * 4) == 0 and n > 0                # parts of a shared contraction
    for kw, d_out, bad in ((dict(d=1000), 256, b.SKIP_ERR_UNSUPPORTED), ({}, 12, b.SKIP_ERR_UNSUPPORTED),
                           ({}, 0, b.SKIP_ERR_INVALID_ARG), ({}, 65544, b.SKIP_ERR_UNSUPPORTED),
                           (dict(d=65568), 8, b.SKIP_ERR_UNSUPPORTED),
                           (dict(dtype="f32"), 256, b.SKIP_ERR_UNSUPPORTED)):
        for f in (b.packed_bytes_dense, b.workspace_bytes_dense):
            with pytest.raises(b.SkipError) as e:
                f(problem(b, **kw), d_out)
            assert e.value.status == bad, (kw, d_out)


def test_pack_refusals(b):
    p = problem(b)

    def call(W=FAKE, d_out=256, packed=FAKE, n=1 << 40, p=p):
        return b.LIB.skip_pack_dense(ctypes.byref(p), W, d_out, packed, n, None)
    inv = b.SKIP_ERR_INVALID_ARG
    assert call(W=None) == inv and call(packed=None) == inv
    assert call(W=FAKE + 8) == inv and call(packed=FAKE + 8) == inv
    assert call(n=256 * 1024 * 2 - 1) == b.SKIP_ERR_WORKSPACE
    assert call(d_out=4) == b.SKIP_ERR_UNSUPPORTED


def test_layer_refusals(b):
    def call(p, n=1 << 40, **kw):
        a = dict(rows=FAKE, ko=FAKE, ri=None, packed=FAKE, d_out=256, bias=None, act=0, res=None,
                 si=None, Y=FAKE, f32=0, ws=FAKE)
        a.update(kw)
        return b.LIB.skip_gather_dense(p and ctypes.byref(p), a["rows"], a["ko"], a["ri"],
                                       a["packed"], a["d_out"], a["bias"], a["act"], a["res"],
                                       a["si"], a["Y"], a["f32"], a["ws"], n, None)
    inv, uns = b.SKIP_ERR_INVALID_ARG, b.SKIP_ERR_UNSUPPORTED
    p = problem(b)
    assert call(None) == inv
    for kw in (dict(rows=None), dict(packed=None), dict(Y=None), dict(f32=2), dict(act=-1),
               dict(act=4), dict(si=FAKE), dict(ri=FAKE, ko=None), dict(rows=FAKE + 2),
               dict(bias=FAKE + 4), dict(res=FAKE + 8), dict(Y=FAKE + 4), dict(ws=FAKE + 8),
               dict(d_out=-8)):
        assert call(p, **kw) == inv, kw
    assert call(problem(b, N=90), ri=FAKE) == inv                   # more kept than tokens
    assert call(problem(b, N=90), res=FAKE, si=FAKE) == inv
    assert call(p, d_out=20) == uns and call(problem(b, d=1016)) == uns
    long = problem(b, d=16384, kept_offsets=[0, 1, 2])
    assert call(long, ws=None) == inv
    assert call(long, n=16) == b.SKIP_ERR_WORKSPACE
    # no rows: nothing to do
    assert call(problem(b, kept_offsets=[0, 0, 0]), rows=None, Y=None, ws=None, n=0) == b.SKIP_OK
    with pytest.raises(KeyError):
        b.ACTIVATIONS["tanh"]
