"""act(W x + b) + residual against float64, over row counts that change the form,
odd widths, indices, activations, in place."""
import math
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_25422_amd import binding
    return binding


def act64(y, name):
    if name == "relu":
        return y.clamp_min(0)
    if name == "gelu":
        return 0.5 * y * (1 + torch.erf(y / math.sqrt(2)))
    if name == "silu":
        return y / (1 + torch.exp(-y))
    return y


def inputs(M, d, d_out, seed, integers=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if integers:                                  # sums are exact in float32
        x = torch.randint(-3, 4, (M, d), generator=g, device="cuda").bfloat16()
        W = torch.randint(-3, 4, (d_out, d), generator=g, device="cuda").bfloat16()
    else:
        x = torch.randn(M, d, generator=g, device="cuda").bfloat16()
        W = (torch.randn(d_out, d, generator=g, device="cuda") / math.sqrt(d)).bfloat16()
    b = torch.randn(d_out, generator=g, device="cuda")
    R = torch.randn(M, d_out, generator=g, device="cuda").bfloat16()
    return x, W, b, R


def problem(B, M, d, N=0, ko=None):
    return B.make_problem("bf16", B=1 if ko is None else len(ko) - 1, N=N, d=d,
                          kept_offsets=[0, M] if ko is None else ko)


def check(Y, x, W, b, R, act):
    """Products are exact and summed in float32, at most d + 2 roundings of the sum
    of magnitudes; the slope of an activation is below 1.13 and its own error a few
    units of its argument and value (2^-20); one rounding to the output's type."""
    x, W = x.double(), W.double()
    y = x @ W.t()
    mag = x.abs() @ W.abs().t()
    if b is not None:
        y = y + b.double()
        mag = mag + b.double().abs()
    pre = act64(y, act)
    want = pre + (R.double() if R is not None else 0)
    tol = 1.13 * 2.0 ** -24 * (x.shape[1] + 2) * mag + 2.0 ** -24 * want.abs()
    if act in ("gelu", "silu"):
        tol = tol + 2.0 ** -20 * (pre.abs() + 2.0 ** -4)
    if Y.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs()
    over = ((Y.double() - want).abs() - tol).max().item()
    print(f"dense {tuple(Y.shape)} d={x.shape[1]} {act} {Y.dtype}: excess {over:.2e}",
          file=sys.stderr, flush=True)
    assert over <= 0


@pytest.mark.parametrize("M", [1, 31, 33, 64, 95, 97, 130, 200, 257, 700])
@pytest.mark.parametrize("d,d_out", [(32, 8), (96, 264), (1408, 520), (4096, 72)])
def test_shapes(B, M, d, d_out):
    x, W, b, R = inputs(M, d, d_out, M + d)
    p = problem(B, M, d)
    packed = B.pack_dense(p, W)
    for act, bias, res, f32 in (("none", None, None, True), ("gelu", b, R, False),
                                ("silu", None, R, True), ("relu", b, None, False)):
        Y = B.gather_dense(p, x, packed, d_out, bias=bias, activation=act, residual=res,
                           out_f32=f32)
        torch.cuda.synchronize()
        check(Y, x, W, bias, res, act)


@pytest.mark.parametrize("M,d,d_out", [(3, 16384, 1024), (291, 16384, 520), (97, 8192, 4104),
                                       (1300, 2048, 2048), (2305, 64, 8200), (5000, 96, 1000)])
def test_larger(B, M, d, d_out):
    """Shared contractions and tall tiles."""
    x, W, b, R = inputs(M, d, d_out, 3)
    p = problem(B, M, d)
    Y = B.gather_dense(p, x, B.pack_dense(p, W), d_out, bias=b, activation="silu", residual=R,
                       out_f32=True)
    torch.cuda.synchronize()
    check(Y, x, W, b, R, "silu")


@pytest.mark.parametrize("M", [1, 33, 96, 97, 161, 193, 225, 500])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 544, 2080])
def test_integers_are_exact(B, M, d):
    """Every step count of the pipelines, on sums that float32 holds."""
    d_out = 328
    x, W, _, _ = inputs(M, d, d_out, d, integers=True)
    p = problem(B, M, d)
    Y = B.gather_dense(p, x, B.pack_dense(p, W), d_out, out_f32=True)
    torch.cuda.synchronize()
    assert torch.equal(Y.double(), x.double() @ W.double().t())


@pytest.mark.parametrize("ks", [[40, 0, 9], [1, 1, 1], [0, 150, 77]])
def test_rows_and_residual_through_indices(B, ks):
    N, d, d_out = 200, 64, 136
    g = torch.Generator().manual_seed(5)
    ko = np.concatenate([[0], np.cumsum(ks)])
    M = int(ko[-1])
    V = torch.randn(3, N, d, generator=g).bfloat16().cuda()
    S = torch.randn(3, N, d_out, generator=g).bfloat16().cuda()
    idx = torch.cat([torch.randperm(N, generator=g)[:k].sort().values for k in ks]).int().cuda()
    own = torch.repeat_interleave(torch.arange(3), torch.tensor(ks)).cuda()
    _, W, b, R = inputs(M, d, d_out, 6)
    p = problem(B, M, d, N, ko)
    packed = B.pack_dense(p, W)
    kod = torch.from_numpy(ko.astype(np.int32)).cuda()
    rows = V[own, idx.long()]
    for ri, si in ((idx, None), (None, idx), (idx, idx)):
        Y = B.gather_dense(p, V if ri is not None else rows, packed, d_out, kod, rows_idx=ri,
                           bias=b, residual=S if si is not None else R, residual_idx=si)
        torch.cuda.synchronize()
        check(Y, rows, W, b, S[own, idx.long()] if si is not None else R, "none")


@pytest.mark.parametrize("M,d,d_out", [(5, 64, 40), (150, 64, 264), (300, 8192, 264),
                                       (2, 8192, 64)])
def test_in_place_residual(B, M, d, d_out):
    x, W, b, R = inputs(M, d, d_out, 7)
    p = problem(B, M, d)
    Y = R.clone()
    B.gather_dense(p, x, B.pack_dense(p, W), d_out, bias=b, residual=Y, out=Y)
    torch.cuda.synchronize()
    check(Y, x, W, b, R, "none")


@pytest.mark.parametrize("M", [7, 250])
def test_rows_past_the_last_stay(B, M):
    x, W, b, _ = inputs(M, 64, 72, 8)
    p = problem(B, M, 64)
    out = torch.full((M + 3, 72), 7.0, device="cuda")
    B.gather_dense(p, x, B.pack_dense(p, W), 72, bias=b, out=out)
    torch.cuda.synchronize()
    assert (out[M:] == 7.0).all()
    check(out[:M], x, W, b, None, "none")


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_activation_tails(B, act):
    """A row of one's bias alone: arguments from -40 to 40, infinite ones too."""
    d_out = 2048
    x, W, _, _ = inputs(1, 32, d_out, 9)
    W.zero_()
    b = torch.linspace(-40, 40, d_out, device="cuda")
    b[0], b[-1] = -1e30, 1e30
    p = problem(B, 1, 32)
    Y = B.gather_dense(p, x, B.pack_dense(p, W), d_out, bias=b, activation=act, out_f32=True)
    torch.cuda.synchronize()
    want = act64(b.double(), act)
    assert torch.isfinite(Y).all()
    # a few units of the value, and of the argument's own rounding in the tails
    tol = 2.0 ** -20 * (want.abs() + 2.0 ** -4)
    assert ((Y[0].double() - want).abs() <= tol).all()


def test_bitwise_repeatable(B):
    x, W, b, R = inputs(300, 8192, 264, 10)
    p = problem(B, 300, 8192)
    packed = B.pack_dense(p, W)
    a = B.gather_dense(p, x, packed, 264, bias=b, residual=R)
    for _ in range(3):
        assert torch.equal(a, B.gather_dense(p, x, packed, 264, bias=b, residual=R))


@pytest.mark.parametrize("M", [2, 40, 200])
@pytest.mark.parametrize("act", ["none", "gelu", "silu", "relu"])
def test_infinities_and_nan(B, M, act):
    """One term a sum, so an infinity or NaN of a row reaches the result as itself:
    infinity, NaN, and below zero the activations' limits (a number times exp(-inf)
    may be no number, as in the formula x / (1 + exp(-x)))."""
    W = torch.zeros(40, 64, dtype=torch.bfloat16, device="cuda")
    W[:, 5] = 1
    x = torch.zeros(M, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 5], x[1, 5] = math.inf, math.nan
    p = problem(B, M, 64)
    Y = B.gather_dense(p, x, B.pack_dense(p, W), 40, activation=act, out_f32=True)
    torch.cuda.synchronize()
    assert (Y[0] == math.inf).all() and Y[1].isnan().all() and not Y[2:].any()
