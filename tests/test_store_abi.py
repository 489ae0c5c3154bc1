"""Refusals of the calls around the 4-bit store, on the host: every call here
fails validation before anything is enqueued."""
import ctypes

import numpy as np
import pytest

FAKE = 1 << 40   # never dereferenced


@pytest.fixture(scope="module")
def b():
    from paper_2607_25422_amd import binding
    return binding


def problem(b, **kw):
    base = dict(B=2, N=576, d=1024, H=16, d_h=64, kept_offsets=[0, 96, 192],
                passage_offsets=[0, 10, 20, 30], query_passages=[0, 2, 3], sm_scale=0.125)
    dtype = kw.pop("dtype", "bf16")
    base.update(kw)
    return b.make_problem(dtype, **base)


def store(b, heads_kv=4, n_blocks=8, data=FAKE, reserved=0):
    return b.SkipKvStore(heads_kv, reserved, n_blocks, data)


def test_struct_and_size(b):
    assert ctypes.sizeof(b.SkipKvStore) == 24 and b.SkipKvStore.data.offset == 16
    assert b.store_bytes(8, 128, 3) == 3 * 8 * 34 * 128
    assert b.store_bytes(1, 64, 0) == 0
    for bad in ((0, 64, 1), (1, 64, -1), (1, 128, 1 << 62)):
        with pytest.raises(b.SkipError) as e:
            b.store_bytes(*bad)
        assert e.value.status == b.SKIP_ERR_INVALID_ARG
    with pytest.raises(b.SkipError) as e:
        b.store_bytes(1, 96, 1)
    assert e.value.status == b.SKIP_ERR_UNSUPPORTED


def test_passage_blocks(b):
    first, end = b.passage_blocks([0, 1, 33, 65, 165], first=3)
    assert first.tolist() == [3, 4, 5, 6] and end == 10 and first.dtype == np.int32
    assert b.passage_blocks([0]) [1] == 0


BAD_STORES = [dict(heads_kv=0), dict(heads_kv=5), dict(reserved=1), dict(n_blocks=-1),
              dict(n_blocks=0), dict(data=None), dict(data=FAKE + 8)]


@pytest.mark.parametrize("fn", ["skip_quantize_passages", "skip_dequantize_passages"])
def test_store_calls(b, fn):
    def call(p, st, **kw):
        a = dict(K=FAKE, V=FAKE, off=FAKE, blk=FAKE, keys=None)
        a.update(kw)
        if fn == "skip_quantize_passages":
            return b.LIB.skip_quantize_passages(p and ctypes.byref(p), st and ctypes.byref(st),
                                                a["K"], a["V"], a["off"], a["blk"], a["keys"],
                                                None)
        return b.LIB.skip_dequantize_passages(p and ctypes.byref(p), st and ctypes.byref(st),
                                              a["off"], a["blk"], a["K"], a["V"], None)
    p = problem(b)
    inv, uns = b.SKIP_ERR_INVALID_ARG, b.SKIP_ERR_UNSUPPORTED
    assert call(None, store(b)) == inv and call(p, None) == inv
    for kw in BAD_STORES:
        assert call(p, store(b, **kw)) == inv, kw
    for kw in (dict(K=None), dict(V=None), dict(off=None), dict(blk=None), dict(K=FAKE + 4),
               dict(V=FAKE + 2)):
        assert call(p, store(b), **kw) == inv, kw
    if fn == "skip_quantize_passages":
        assert call(p, store(b), keys=FAKE + 4) == inv
    assert call(problem(b, d=1280, H=16, d_h=80), store(b)) == uns
    assert call(problem(b, d=1024, H=4, d_h=64), store(b)) == inv       # H * d_h != d
    assert call(problem(b, passage_offsets=[0, 10, 20, 300]), store(b)) == inv   # does not fit
    q = problem(b)
    q.L_max = 0
    assert call(q, store(b)) == inv
    q = problem(b)
    q.dtype = 3
    assert call(q, store(b)) == inv
    # nothing to do
    empty = problem(b, passage_offsets=[0], query_passages=[0, 0, 0])
    assert call(empty, store(b, n_blocks=0, data=None), K=None, V=None, off=None,
                blk=None) == b.SKIP_OK


def xattn(b, p, st, ws_bytes=1 << 40, **kw):
    names = ("rows", "ko", "idx", "erows", "po", "pb", "qp", "keys", "keep", "rp", "col", "O",
             "lse", "rpo", "colo", "ws")
    a = dict(rows=FAKE, ko=FAKE, idx=None, erows=None, po=FAKE, pb=FAKE, qp=FAKE, keys=FAKE,
             keep=None, rp=None, col=None, O=FAKE, lse=None, rpo=None, colo=None, ws=FAKE)
    a.update(kw)
    return b.LIB.skip_bipartite_xattn_quant(ctypes.byref(p), ctypes.byref(st),
                                            *[a[n] for n in names], ws_bytes, None)


def test_attention_refusals(b):
    p, st = problem(b), store(b)
    inv, uns = b.SKIP_ERR_INVALID_ARG, b.SKIP_ERR_UNSUPPORTED
    for kw in BAD_STORES:
        assert xattn(b, p, store(b, **kw)) == inv, kw
    for kw in (dict(rows=None), dict(ko=None), dict(po=None), dict(pb=None), dict(qp=None),
               dict(keys=None), dict(O=None), dict(ws=None), dict(rows=FAKE + 2),
               dict(erows=FAKE + 8), dict(O=FAKE + 4), dict(keys=FAKE + 4), dict(ws=FAKE + 8),
               dict(rpo=FAKE), dict(colo=FAKE), dict(col=FAKE),
               dict(rp=FAKE, rpo=FAKE, colo=FAKE), dict(rp=FAKE, erows=FAKE),
               dict(rp=FAKE, keep=FAKE)):
        assert xattn(b, p, st, **kw) == inv, kw
    q = problem(b, total_edges=3)
    assert xattn(b, q, st, rp=FAKE) == inv                              # edges without columns
    assert xattn(b, problem(b, N=90), st, idx=FAKE) == inv              # more kept than tokens
    assert xattn(b, problem(b, dtype="f32"), st) == uns
    assert xattn(b, problem(b, d=4096, H=64), store(b, heads_kv=1)) == uns   # 64 query heads
    assert xattn(b, problem(b, query_passages=[0, 0, 65],
                            passage_offsets=list(range(66))), st) == uns
    for bad in (float("inf"), float("nan")):
        assert xattn(b, problem(b, sm_scale=bad), st) == inv
    need = ctypes.c_size_t(0)
    assert b.LIB.skip_workspace_bytes_quant(ctypes.byref(p), ctypes.byref(st),
                                            ctypes.byref(need)) == b.SKIP_OK
    assert need.value > 0
    assert xattn(b, p, st, ws_bytes=need.value - 1) == b.SKIP_ERR_WORKSPACE
    assert b.LIB.skip_workspace_bytes_quant(ctypes.byref(p), ctypes.byref(st), None) == inv
    assert b.LIB.skip_workspace_bytes_quant(None, ctypes.byref(st), ctypes.byref(need)) == inv
    # no rows: nothing to do
    none = problem(b, kept_offsets=[0, 0, 0])
    assert xattn(b, none, st, rows=None, O=None) == b.SKIP_OK
