"""Rotations by any finite frequency at any position, against angles in whole numbers.

An angle is held to 2^-31 of a turn; its sine and cosine are polynomials in fp32 (argument, steps and result: 2^-22 with the
next terms), and a rotated channel is two products: 2^-21 (|a| + |b|) in all."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from test_gpu_token_steps import dev, draw, host, i32, nan

pytestmark = pytest.mark.gpu

DIGITS = 1400


def arctan_inverse(x, one):
    """one * arctan(1 / x), by its series."""
    term = total = one // x
    k = 1
    while term:
        term //= -x * x
        k += 2
        total += term // k
    return total


ONE = 1 << (DIGITS + 64)
PI = 4 * (4 * arctan_inverse(5, ONE) - arctan_inverse(239, ONE))


def turns(freq, position):
    """freq * position / 2 pi modulo 1, to some 300 digits at the largest."""
    f = Fraction(freq) * position
    return float(Fraction(f.numerator * ONE % (2 * PI * f.denominator), 2 * PI * f.denominator))


def test_turns():
    assert abs(PI / ONE - math.pi) < 1e-15 and abs(turns(1.0, 3) - 3 / (2 * math.pi)) < 1e-15
    assert abs(turns(-0.5, 1) - (1 - 0.5 / (2 * math.pi))) < 1e-15


FREQS = [1.0, 0.1, -0.3, 100.0, -77.7, 1e4, 12345.678, -1e6, 3.7e9, 1e15, 2.0 ** 53 + 2, -2.0 ** 64, 1e25, 6.02e100, -1.7e308, 5e-324]


@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_heads_angles_of_any_frequency(layout):
    from paper_2406_02052_amd import HeadNorm

    n, pairs = 64, len(FREQS)
    r = np.random.RandomState(1)
    pos = np.concatenate([[0, 1, -1, 7, 2 ** 31 - 1, -2 ** 31, 10 ** 6], r.randint(-2 ** 31, 2 ** 31 - 1, n - 7)])
    q, = draw(2, (1, n, 1, 2 * pairs))
    op = HeadNorm(1, n, 1, 0, 2 * pairs, "fp32", norm=None, layout=layout, freq=FREQS)
    y = nan(q.shape)
    op.forward(dev(q, "fp32"), None, y, None, positions=i32(pos.reshape(1, 1, n)))
    back = nan(q.shape)
    op.backward(None, None, y, None, back, None, positions=i32(pos.reshape(1, 1, n)))
    got, back = host(y), host(back)
    for i, f in enumerate(FREQS):
        a, b = (i, i + pairs) if layout == "halves" else (2 * i, 2 * i + 1)
        t = 2 * math.pi * np.array([turns(f, int(p)) for p in pos])
        u, v = q[0, :, 0, a], q[0, :, 0, b]
        bar = 2.0 ** -21 * (np.abs(u) + np.abs(v))
        assert (np.abs(got[0, :, 0, a] - (u * np.cos(t) - v * np.sin(t))) <= bar).all(), f
        assert (np.abs(got[0, :, 0, b] - (u * np.sin(t) + v * np.cos(t))) <= bar).all(), f
        # turned back
        assert (np.abs(back[0, :, 0, a] - u) <= 3 * bar).all() and (np.abs(back[0, :, 0, b] - v) <= 3 * bar).all(), f
