"""Sizes past the limits of the calls around the 4-bit store and of the layer: refused
on the host, by the workspace queries too, before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2607_25422_amd import binding as B

FAKE = 1 << 40   # never dereferenced


def problem(**kw):
    p = B.SkipProblem()
    p.dtype = B.SKIP_BF16
    p.sm_scale, p.avg_degree = 0.125, 4.0
    for n, v in {**dict(B=1, N=576, H=32, d_h=64, k_max=1, P_max=1, L_max=32), **kw}.items():
        setattr(p, n, v)
    p.d = kw.get("d", p.H * p.d_h)
    p.total_kept = kw.get("total_kept", p.B * p.k_max)
    p.total_passages = kw.get("total_passages", p.B * p.P_max)
    p.total_tokens = kw.get("total_tokens", p.total_passages * p.L_max)
    return p


def attend(p, heads_kv, given, n_blocks=8):
    """(workspace query, call) of the attention, the graph given or built."""
    st = B.SkipKvStore(heads_kv, 0, n_blocks, FAKE)
    n = ctypes.c_size_t(0)
    a = B.LIB.skip_workspace_bytes_quant(ctypes.byref(p), ctypes.byref(st), ctypes.byref(n))
    graph = [FAKE, FAKE] if given else [None, None]
    out = [None, None] if given else [FAKE, FAKE]
    p.total_edges = p.total_kept if given else 0
    b = B.LIB.skip_bipartite_xattn_quant(
        ctypes.byref(p), ctypes.byref(st), FAKE, FAKE, None, None, FAKE, FAKE, FAKE,
        None if given else FAKE, None, *graph, FAKE, None, *out, FAKE, 1 << 50, None)
    return a, b


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("kw,heads_kv", [
    (dict(B=131100), 32),                            # 4 195 200 workgroups of one row
    (dict(B=4096, k_max=6145, total_kept=20000, N=8192), 32),    # 33 chunks of the longest
])
def test_too_many_workgroups_of_the_attention(kw, heads_kv, given):
    assert attend(problem(**kw), heads_kv, given) == (B.SKIP_ERR_UNSUPPORTED,) * 2


def test_the_largest_grid_of_the_attention_has_a_workspace():
    st = B.SkipKvStore(32, 0, 8, FAKE)
    n = ctypes.c_size_t(0)
    for kw in (dict(B=131072), dict(B=4096, k_max=6144, total_kept=30000, N=8192)):
        assert B.LIB.skip_workspace_bytes_quant(ctypes.byref(problem(**kw)), ctypes.byref(st),
                                                ctypes.byref(n)) == B.SKIP_OK


def test_too_many_tiles_of_the_layer():
    def call(M, d_out):
        p = problem(H=1, d=64, total_kept=M)
        n = ctypes.c_size_t(0)
        a = B.LIB.skip_workspace_bytes_dense(ctypes.byref(p), d_out, ctypes.byref(n))
        return a, lambda: B.LIB.skip_gather_dense(
            ctypes.byref(p), FAKE, FAKE, None, FAKE, d_out, None, 0, None, None, FAKE, 0, FAKE,
            1 << 50, None)
    a, b = call(1 << 23, 65536)                      # 8 388 608 x 65536: 2^23 tiles at least
    assert a == b() == B.SKIP_ERR_UNSUPPORTED
    assert call(1 << 20, 65536)[0] == B.SKIP_OK


def test_token_numbers_near_the_end_of_32_bits():
    """2^31 - 128 tokens are taken, more refused (by the same check as a passage that
    does not fit its store, whose count of records must not wrap)."""
    inv, uns = B.SKIP_ERR_INVALID_ARG, B.SKIP_ERR_UNSUPPORTED
    top = (1 << 31) - 128
    for n, n_blocks, want in ((top, top // 32, B.SKIP_OK), (top, top // 32 - 1, inv), (top, 1, inv),
                              (top + 1, 1, uns), ((1 << 31) - 1, 1, uns),
                              ((1 << 31) - 1, 1 << 26, uns)):
        p = problem(H=1, L_max=n)
        st = B.SkipKvStore(1, 0, n_blocks, FAKE)
        size = ctypes.c_size_t(0)
        assert B.LIB.skip_workspace_bytes_quant(ctypes.byref(p), ctypes.byref(st),
                                                ctypes.byref(size)) == want, (n, n_blocks)
        if want != B.SKIP_OK:
            assert B.LIB.skip_quantize_passages(ctypes.byref(p), ctypes.byref(st), FAKE, FAKE,
                                                FAKE, FAKE, None, None) == want
            assert B.LIB.skip_dequantize_passages(ctypes.byref(p), ctypes.byref(st), FAKE, FAKE,
                                                  FAKE, FAKE, None) == want


def test_blocks_of_a_passage():
    """The blocks that the store's kernels visit go by the batch's longest passage: those
    past a shorter one's end are none of its, also where their token number would pass
    32 bits."""
    f = B.LIB["_ZN4skip11store_blockEiiiRi"]
    f.restype, f.argtypes = ctypes.c_bool, [ctypes.c_int] * 3 + [ctypes.POINTER(ctypes.c_int)]
    top = (1 << 31) - 128
    cases = [(0, 0), (5, 5), (0, 1), (7, 39), (7, 40), (100, 197), (0, top), (top - 40, top),
             (1 << 30, (1 << 30) + 33), (top, top)]
    for ts, te in cases:
        for i in {0, 1, 2, 3, 1 << 24, (1 << 25) + 2, (top - 1) // 32}:
            t0 = ctypes.c_int(-1)
            got = f(ts, te, i, ctypes.byref(t0))
            assert got == (ts + 32 * i < te), (ts, te, i)
            assert not got or t0.value == ts + 32 * i


@pytest.mark.parametrize("shape", [(8, 96), (8, 32), (64,), (8, 2, 64)])
def test_weights_of_another_width_are_refused(shape):
    """Wider rows would be packed as rows of the problem's width."""
    p = B.make_problem("bf16", B=1, d=64, kept_offsets=[0, 1])
    with pytest.raises(ValueError, match="W must be"):
        B.skip_pack_dense(p, torch.zeros(shape, dtype=torch.bfloat16),
                          torch.empty(1 << 16, dtype=torch.uint8))
