"""Softmax weights and sums of the attention over the 4-bit store at the ends of
their ranges."""
import math

import numpy as np
import pytest
import torch

from test_gpu_store import Held, attend, check, cum, dev, reference, say

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
