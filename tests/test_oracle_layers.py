"""Pins of the plain definitions of the single integer layers: against exact fractions and real arithmetic."""
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import layers as P


@pytest.mark.parametrize("s", [0, 1, 7, 31])
def test_requantisation_rounds_half_up(s):
    rng = np.random.default_rng(s)
    a = np.concatenate([rng.integers(-2 ** 31, 2 ** 31, 200), [0, 1, -1, 2 ** 31 - 1, -2 ** 31]])
    m = rng.integers(-2 ** 31 + 1, 2 ** 31, a.size)
    got = P.rq(a, m, np.full(a.size, s))
    for x, y, g in zip(a, m, got):
        assert g == math.floor(Fraction(int(x) * int(y), 2 ** (31 + s)) + Fraction(1, 2))


def test_a_norm_of_ones_is_the_reciprocal_root():
    # D = C + eps; the value is 2^22 / sqrt(D) but for the two floors and one rounding
    for C, eps in ((1, 1), (4, 12), (173, 1), (4096, 10 ** 6)):
        got = P.normed_row([1] * C, "rms", eps)[0]
        assert abs(got - 2.0 ** 22 / math.sqrt(C + eps)) < 0.51


@pytest.mark.parametrize("kind", ["rms", "centred"])
def test_norm_follows_real_arithmetic(kind):
    rng = np.random.default_rng(3)
    for scale in (1, 30, 5000, 2 ** 23):
        v = np.clip(np.round(rng.normal(0, scale, (4, 61)) + scale / 3), -2 ** 23, 2 ** 23 - 1).astype(np.int64)
        x = v.astype(np.float64)
        if kind == "centred":
            x = x - np.floor(x.mean(1) + 0.5)[:, None]
        want = x * 2.0 ** 22 / np.sqrt((x * x).sum(1) + 5)[:, None]
        # sigma and rho are floors of numbers of at least 2^30: two relative errors of 2^-30, then half a unit
        assert np.abs(P.normed(v, kind, 5) - want).max() <= 0.5 + 2.0 ** 22 * 3 * 2.0 ** -30


def test_a_norm_of_zeros_and_of_the_widest_values():
    assert P.normed_row([0, 0, 0], "rms", 1) == [0, 0, 0]
    assert P.normed_row([7, 7, 7], "centred", 1) == [0, 0, 0]
    top = P.normed_row([-2 ** 31] * 8192, "rms", 1 << 60)          # taken as -2^23
    D = 2 ** 46 * 8192 + 2 ** 60
    assert abs(top[0] + 2 ** 45 / math.sqrt(D)) < 0.6
    assert max(abs(e) for e in P.normed_row([2 ** 23 - 1], "rms", 1)) <= 2 ** 22 + 1


def test_adapters_are_further_input_channels():
    """A projection with an adapter equals the one of a layer with rank more input channels fed with h."""
    rng = np.random.default_rng(1)
    K, N, R, rows = 9, 5, 3, 7
    layer = {"k": 1, "c_in": K, "c_out": N, "w": rng.integers(-127, 128, (N, K)).astype(np.int8),
             "bias": rng.integers(-999, 999, N).astype(np.int32), "m0": rng.integers(2 ** 30, 2 ** 31, N),
             "s": np.full(N, 5), "relu": True, "clamp": (0, 255)}
    ad = {"rank": R, "down": rng.integers(-127, 128, (R, K)).astype(np.int8), "m0": rng.integers(2 ** 30, 2 ** 31, R),
          "s": np.full(R, 6), "up": rng.integers(-127, 128, (N, R)).astype(np.int8)}
    x = rng.integers(0, 256, (rows, K)).astype(np.uint8)
    h = np.clip(P.rq(x.astype(np.int64) @ ad["down"].astype(np.int64).T, ad["m0"], ad["s"]), -128, 127)
    wide = dict(layer, c_in=K + R, w=np.concatenate([layer["w"], ad["up"]], 1))
    y = np.full((rows, N), -9)
    got = P.projection(layer, x, [ad], [0, 4, 6], [0, -1], y)
    np.testing.assert_array_equal(got[:4], P.projection(wide, np.concatenate([x, h], 1))[:4])
    np.testing.assert_array_equal(got[4:6], P.projection(layer, x)[4:6])
    assert (got[6:] == -9).all()
