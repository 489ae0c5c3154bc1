"""The oracle of the 4-bit store against worked examples and enumeration."""
import itertools
import math

import numpy as np

import oracle as orc

GRID = sorted({s * v for v in (0, .5, 1, 1.5, 2, 3, 4, 6) for s in (-1, 1)})


def test_worked_block():
    # max 6: the least power of two with 6 <= 7 * 2^e is 1; ties at .25, .75, ..
    x = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.2, -0.3, -5.01, 0, 4.99, 2.51, 1.74, 0.76]
    codes, s, v = orc.held_block(x)
    assert s == 127
    assert v.tolist() == [6, 4, 4, 2, 2, 1, 1, 0, 0, -.5, -6, 0, 4, 3, 1.5, 1]
    assert codes[:3] == [7, 6, 6] and codes[8] == 8


def test_scale_is_the_least_whose_seven_reaches_the_maximum():
    for a, e in ((7.0, 0), (np.nextafter(7.0, 8), 1), (3.5, -1), (3.6, 0), (1.75 * 2 ** 100, 98),
                 (2.0 ** -140, -126), (0.0, -126)):
        assert orc.held_block([a, 0.0])[1] == e + 127, a


def test_every_value_is_a_nearest_one():
    rng = np.random.default_rng(3)
    for _ in range(50):
        x = rng.standard_normal(32) * 2.0 ** rng.integers(-20, 20)
        _, s, v = orc.held_block(x)
        p = 2.0 ** (s - 127)
        for a, b in zip(x, v):
            assert abs(a - b) == min(abs(a - g * p) for g in GRID)
        # half a step at most: 1 up to 7 (in units of the power of two)
        assert np.max(np.abs(x - v)) <= p


def test_held_values_are_held_as_they_are():
    for s, c in itertools.product((-30, 0, 30), range(4)):
        x = np.array([6.0 if c == 0 else 4.0, -3, 1.5, .5, 0, 1, -2, 4]) * 2.0 ** s
        assert orc.held_block(x)[2].tolist() == x.tolist()


def test_passage_blocks():
    rng = np.random.default_rng(4)
    K, V = rng.standard_normal((35, 1, 64)), rng.standard_normal((35, 1, 64))
    Ko, Vo = orc.held_passage(K, V)
    assert Ko[34, 0, 32:].tolist() == orc.held_block(K[34, 0, 32:])[2].tolist()
    assert Vo[32:, 0, 7].tolist() == orc.held_block(V[32:, 0, 7])[2].tolist()
    assert Vo[:32, 0, 7].tolist() == orc.held_block(V[:32, 0, 7])[2].tolist()
    assert math.isfinite(float(Ko.sum() + Vo.sum()))


def test_the_largest_values_are_held_as_finite_ones():
    top = 6.0 * 2.0 ** 125
    x = [math.inf, -math.inf, 3.4e38, -1.8 * 2.0 ** 127, 2.0 ** 127, 0.0]
    _, s, v = orc.held_block(x)
    assert s == 252 and v.tolist() == [top, -top, top, -top, 2.0 ** 127, 0.0]
