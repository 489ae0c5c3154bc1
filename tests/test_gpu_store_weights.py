"""Softmax weights and sums of the attention over the 4-bit store at the ends of
their ranges."""
import math

import numpy as np
import pytest
import torch

from test_gpu_store import Held, attend, check, cum, dev, reference, rows_of, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2607_25422_amd import binding
    return binding


def batch(x, Ls, nq):
    """The same stored passages for each of nq questions (1: the form of few rows; 200
    of 4 heads: that of many)."""
    x.off, x.po = cum(Ls * nq), dev(cum(Ls * nq))
    x.pb = dev(np.tile(x.blocks, nq))


@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("o_f32", [False, True])
def test_rising_logits_over_the_largest_values(B, nq, D, o_f32):
    """Logits of log2 0, then 7.875 in one tile, then 15.75 in thousands of tokens: a
    reference may lag in a passage, and again where passages are merged.  Every value
    is the largest held one, so the result is that value."""
    H, Ls, n = 4, [40, 4096], 3
    x = Held(B, Ls, H, H, D, 62)
    x.K, x.V = torch.zeros_like(x.K), torch.full_like(x.V, 6 * 2.0 ** 125)
    x.V[:, :, 1::2] *= -1
    x.K[40:104, :, 5], x.K[104:, :, 5] = 1.0, 2.0
    Q = torch.zeros(n, H, D).bfloat16()
    Q[:, :, 5] = 7.875
    x.write(B)
    V = x.V.double().numpy()                 # held as they are
    batch(x, Ls, nq)
    nb = [[0, 1], [1], [0, 1]]
    say(f"rising logits nq={nq} D={D} f32={o_f32}")
    O, lse = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [n] * nq, [2] * nq, math.log(2), o_f32)
    torch.cuda.synchronize()
    O, lse = O.view(nq, n, H, D), lse.view(nq, n, H)
    assert (O == O[:1]).all() and (lse == lse[:1]).all()
    ref = reference(Q.double().numpy(), x.K.double().numpy(), V, nb, [n], [2], cum(Ls),
                    math.log(2), 1, o_f32)
    check(O[0], lse[0], ref, o_f32, "rising logits")


@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("o_f32", [False, True])
def test_weights_of_averages_that_cancel(B, nq, D, o_f32):
    """Two tokens of values a and -b, their weights b to a as near as a query of three
    bf16 features says it: the average is near 0, so that a bf16 output has steps far
    below a weight's error of 2^-16 of itself (the bound of `reference`, which takes
    the values' magnitude for the size of that error)."""
    H = 4
    pairs = [(3.0, 1.0), (3.0, 2.0), (6.0, 1.0), (6.0, 4.0), (6.0, 0.5), (1.5, 0.5)]
    Ls, n = [2] * len(pairs), len(pairs)
    x = Held(B, Ls, H, H, D, 61)
    x.K, x.V = torch.zeros_like(x.K), torch.zeros_like(x.V)
    x.K[0::2, :, :3] = 1.0
    Q = torch.zeros(n, H, D)
    for i, (a, b) in enumerate(pairs):
        x.V[2 * i], x.V[2 * i + 1] = a, -b
        z = math.log(b / a)
        for f in range(3):
            Q[i, :, f] = torch.tensor(z).bfloat16().float()
            z -= float(Q[i, 0, f])
    Q = Q.bfloat16()
    x.write(B)
    K, V = x.held1()
    assert np.array_equal(K, x.K.double().numpy()) and np.array_equal(V, x.V.double().numpy())
    batch(x, Ls, nq)
    nb = [[i] for i in range(n)]
    say(f"weights of averages that cancel nq={nq} D={D} f32={o_f32}")
    O, lse = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [n] * nq, [n] * nq, 1.0, o_f32)
    torch.cuda.synchronize()
    O, lse = O.view(nq, n, H, D), lse.view(nq, n, H)
    assert (O == O[:1]).all() and (lse == lse[:1]).all()
    ref = reference(Q.double().numpy(), K, V, nb, [n], [n], cum(Ls), 1.0, 1, o_f32,
                    piece=2.0 ** -24 if o_f32 else 2.0 ** -16)
    check(O[0], lse[0], ref, o_f32, "cancelling")


@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("D", [64, 128])
def test_zero_features_leave_the_others_as_they_are(B, nq, D):
    """Heads padded by features of zeros: the other features' bits and the LSE are
    those without them."""
    H, Ls, k = 4, [70, 33, 128], 9
    nb = [[0, 2], [1], [], [0, 1, 2], [2], [0], [1, 2], [0, 1], [2]]
    Q = rows_of(k, H, D, 63).repeat(nq, 1, 1)
    got = []
    for pad in (False, True):
        x = Held(B, Ls, H, H, D, 64)
        if pad:
            x.V = x.V.clone()
            x.V[:, :, D // 2:] = 0.0
        x.write(B)
        batch(x, Ls, nq)
        got.append(attend(B, x, Q, nb * nq, [k] * nq, [3] * nq, 0.3))
    torch.cuda.synchronize()
    (O, lse), (P, plse) = got
    assert torch.equal(O[:, :, :D // 2], P[:, :, :D // 2]) and torch.equal(lse, plse)
    assert not P[:, :, D // 2:].any()


@pytest.mark.parametrize("nq", [1, 200])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -121, -2.0 ** -110])
@pytest.mark.parametrize("o_f32", [False, True])
def test_small_scales_of_large_products(B, nq, scale, o_f32):
    """Queries and keys of 2^57: products of 2^120, which a scale brings down to 2^-1,
    2^10 or 0."""
    H, D, Ls, k = 4, 64, [70, 33], 5
    x = Held(B, Ls, H, H, D, 65, make=None)
    x.K = (x.K.float() * 2.0 ** 57).to(x.dt)
    x.write(B)
    Q = (rows_of(k, H, D, 66).float() * 2.0 ** 57).bfloat16()
    batch(x, Ls, nq)
    nb = [[0, 1], [1], [], [0], [0, 1]]
    say(f"small scale {scale} nq={nq} f32={o_f32}")
    O, lse = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [k] * nq, [2] * nq, scale, o_f32)
    torch.cuda.synchronize()
    O, lse = O.view(nq, k, H, D), lse.view(nq, k, H)
    ref = reference(Q.double().numpy(), *x.held1(), nb, [k], [2], cum(Ls), scale, 1, o_f32)
    check(O[0], lse[0], ref, o_f32, "small scale")
    assert (O == O[:1]).all() and (lse == lse[:1]).all()


FORMS = pytest.mark.parametrize("nq,Hkv,Ls", [(1, 1, [40, 2000]),      # split and joined
                                              (3, 4, [40, 90]),        # row tiles
                                              (200, 4, [40, 90])])     # many items


@FORMS
@pytest.mark.parametrize("o_f32", [False, True])
def test_logits_past_float32_weigh_nothing(B, nq, Hkv, Ls, o_f32):
    """A passage whose every product is -2^160: -inf in float32, and of no weight beside
    another passage, whichever comes first."""
    H, D, k = 4, 64, 4
    for order in (0, 1):
        far = slice(0, Ls[0]) if order == 0 else slice(Ls[1], sum(Ls))
        L = Ls if order == 0 else Ls[::-1]
        x = Held(B, L, H, Hkv, D, 67)
        x.K = x.K.clone()
        x.K[:, :, :32] = 0.0
        x.K[far, :, 3] = -2.0 ** 60
        x.write(B)
        Q = rows_of(k, H, D, 68)
        Q[:, :, 3] = 2.0 ** 100
        batch(x, L, nq)
        near = 1 - order
        nb = [[0, 1], [near], [0, 1], []]
        say(f"past float32 nq={nq} Ls={L} f32={o_f32}")
        O, lse = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [k] * nq, [2] * nq, 0.2, o_f32)
        torch.cuda.synchronize()
        O, lse = O.view(nq, k, H, D), lse.view(nq, k, H)
        assert (O == O[:1]).all() and (lse == lse[:1]).all()
        Q = Q.clone()
        Q[:, :, 3] = 0.0                     # (its products with the other passage)
        ref = reference(Q.double().numpy(), *x.held1(), [[near], [near], [near], []], [k], [2],
                        cum(L), 0.2, H // Hkv, o_f32)
        check(O[0], lse[0], ref, o_f32, "past float32")


@FORMS
@pytest.mark.parametrize("o_f32", [False, True])
def test_a_row_that_is_no_number_stays_one(B, nq, Hkv, Ls, o_f32):
    """NaN in, NaN out in every form, and nothing else changes."""
    H, D, k = 4, 64, 5
    x = Held(B, Ls, H, Hkv, D, 69)
    x.write(B)
    batch(x, Ls, nq)
    Q = rows_of(k, H, D, 70)
    nb = [[0, 1], [1], [0, 1], [0], []]
    a = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [k] * nq, [2] * nq, 0.2, o_f32)
    Q[2, 1, 7] = math.nan
    b = attend(B, x, Q.repeat(nq, 1, 1), nb * nq, [k] * nq, [2] * nq, 0.2, o_f32)
    torch.cuda.synchronize()
    for s, t in ((a[0].view(nq, k, H, D).clone(), b[0].view(nq, k, H, D)),
                 (a[1].view(nq, k, H, 1).clone(), b[1].view(nq, k, H, 1))):
        assert t[:, 2, 1].isnan().all()
        s[:, 2, 1] = 0
        t[:, 2, 1] = 0
        assert torch.equal(s, t)
