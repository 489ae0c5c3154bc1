"""Sizes past the limits of the calls around the 4-bit store and of the layer: refused
on the host, by the workspace queries too, before anything is enqueued."""
import ctypes

import pytest

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
