"""Pins for oracle/q8.py: codes by exact fractions, products by loops, the norm by what it has to leave unchanged."""
import math
from fractions import Fraction

import numpy as np

from oracle import q8 as o_q8


def _nearest(f):
    """A fraction to the nearest integer, ties to even."""
    lo = math.floor(f)
    d = f - lo
    return lo + (d > Fraction(1, 2) or (d == Fraction(1, 2) and lo % 2 == 1))


def test_codes_are_the_exact_quotient_rounded():
    rng = np.random.default_rng(3)
    t = rng.standard_normal((40, 33)).astype(np.float32)
    for r in range(40):  # ties and their neighbours: t = (k + 1/2) / 127 of a maximum that 127 divides, and half of any maximum
        top = np.float32(127 * rng.integers(1, 200) / 64) if r % 2 else np.abs(t[r]).max()
        t[r, 0] = top
        t[r, 1:4] = [np.float32(top) / 2, np.nextafter(top / 2, np.float32(0)), -np.nextafter(top / 2, top)]
        k = rng.integers(0, 126, 8) + 0.5
        t[r, 4:12] = (k * (top / 127)).astype(np.float32)
        t[r, 12:] = np.clip(t[r, 12:], -top, top)
    q, s = o_q8.quantise(t)
    for r in range(40):
        top = max(abs(Fraction(float(v))) for v in t[r])
        assert [int(v) for v in q[r]] == [_nearest(127 * Fraction(float(v)) / top) for v in t[r]]
        assert s[r] == float(top) / 127


def test_rows_of_zeros_nan_and_infinity():
    t = np.zeros((4, 3), dtype=np.float32)
    t[1, 1], t[2, 0], t[3] = np.nan, -np.inf, [1e-45, 0, -1e-45]
    q, s = o_q8.quantise(t)
    assert (q[:3] == 0).all() and list(q[3]) == [127, 0, -127] and s[0] == 0 and np.isnan(s[1:3]).all()


def test_norm_scales_a_row_and_leaves_its_codes():
    rng = np.random.default_rng(4)
    x, gain = rng.standard_normal((5, 64)), 1 + 0.1 * rng.standard_normal(64)
    ident = lambda h: h.astype(np.float64)  # noqa: E731
    q, s, h = o_q8.add_norm(x.astype(np.float32), gain.astype(np.float32), None, 1e-30, ident)
    q2, s2, _ = o_q8.add_norm((4 * x).astype(np.float32), gain.astype(np.float32), None, 1e-30, ident)
    assert (q == q2).all() and np.allclose(s, s2, rtol=1e-14)  # (whatever the size of the row)
    y = h / np.sqrt((h ** 2).mean(1, keepdims=True)) * gain
    assert np.abs(q * s[:, None] - y).max() <= 0.5001 * s.max()
    half = (x / 2).astype(np.float32)
    q3, s3, h3 = o_q8.add_norm(half, gain.astype(np.float32), half, 1e-30, ident)
    assert np.array_equal(h3, h) and (q3 == q).all()


def test_product_and_gate():
    rng = np.random.default_rng(5)
    q, c = rng.integers(-128, 128, (3, 7)), rng.integers(-128, 128, (4, 7))
    s, w = rng.random(3), rng.random(4)
    y = o_q8.product(q, s, c, w)
    for m in range(3):
        for n in range(4):
            assert math.isclose(y[m, n], s[m] * w[n] * sum(int(q[m, k]) * int(c[n, k]) for k in range(7)), rel_tol=1e-15)
    z = o_q8.gated(y)
    assert z.shape == (3, 2) and math.isclose(z[1, 1], y[1, 1] / (1 + math.exp(-y[1, 1])) * y[1, 3], rel_tol=1e-14)
    assert o_q8.gated(np.array([[-1e6, 3.0]]))[0, 0] == 0 and o_q8.gated(np.array([[50.0, 2.0]]))[0, 0] == 100
