"""The layer's activations far from zero, relative to their own values, and of
infinities."""
import math
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_25422_amd import binding
    return binding


def activation(B, M, b, act):
    """act(b) in every row, float output: weights of zeros, b the bias."""
    W = torch.zeros(b.numel(), 32, dtype=torch.bfloat16, device="cuda")
    p = B.make_problem("bf16", B=1, d=32, kept_offsets=[0, M])
    x = torch.ones(M, 32, dtype=torch.bfloat16, device="cuda")
    Y = B.gather_dense(p, x, B.pack_dense(p, W), b.numel(), bias=b, activation=act, out_f32=True)
    torch.cuda.synchronize()
    return Y


@pytest.mark.parametrize("M", [1, 40])
def test_gelu_relative(B, M):
    """x / 2 erfc(-x / sqrt 2): the exponent x^2 / 2 log2 e takes three roundings of
    2^-24 at most (of x^2, of the constant, of their product: 2.5 x^2 / 2 of 2^-24 in the
    result, one of them half a step), the polynomial 2.6e-7 = 4.4 of 2^-24, the eleven
    other operations less than one each; down to -8.4, past which the polynomial is not
    fitted (4.5e-5 < 2^-14)."""
    b = torch.linspace(-13, 13, 4096, device="cuda")
    Y = activation(B, M, b, "gelu").double()
    x = b.double()
    want = (x / 2 * torch.special.erfc(-x / math.sqrt(2)))
    bound = (1.25 * x * x * (x < 0) + 16) * 2.0 ** -24
    bound = torch.where(x < -8.4, torch.full_like(x, 2.0 ** -14), bound)
    rel = ((Y - want) / want).abs()
    for lo, hi in ((-13, -8.4), (-8.4, -6), (-6, -2), (-2, 0), (0, 13)):
        at = (x >= lo) & (x < hi)
        print(f"gelu M={M} {lo}..{hi}: {rel[:, at].max().item():.2e}", file=sys.stderr, flush=True)
    assert (rel <= bound).all()


@pytest.mark.parametrize("M", [1, 40])
def test_silu_relative(B, M):
    """x / (1 + exp(-x)): the exponent's two roundings are |x| 2^-23 in the result, the
    other operations a few units."""
    b = torch.linspace(-86, 86, 4096, device="cuda")
    Y = activation(B, M, b, "silu").double()
    x = b.double()
    want = x / (1 + torch.exp(-x))
    rel = ((Y - want) / want).abs()
    print(f"silu M={M}: {rel.max().item():.2e}", file=sys.stderr, flush=True)
    assert (rel <= (2 * x.abs() * (x < 0) + 8) * 2.0 ** -24).all()


@pytest.mark.parametrize("M", [1, 40])
@pytest.mark.parametrize("act", ["relu", "gelu", "none"])
def test_infinities_of_either_sign(B, M, act):
    b = torch.tensor([math.inf, -math.inf, 1e30, -1e30] * 2, device="cuda")
    Y = activation(B, M, b, act)
    want = b if act == "none" else b.clamp_min(0)
    assert torch.equal(Y, want.expand(M, -1))
