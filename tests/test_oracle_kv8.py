"""Pins for oracle/kv8.py: formats by their definition, quantisation by brute force, attention by closed forms."""
import math

import numpy as np
import pytest

from oracle import forward as o_fwd
from oracle import kv8 as o_kv8


def test_code_values():
    import torch

    v = o_kv8.code_values("e4m3")
    assert len(v) == 253 and v[-1] == 448 and v[0] == -448  # 256 codes less two NaN and the second zero
    bits = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert sorted(set(bits[np.isfinite(bits)])) == list(v)
    assert list(o_kv8.code_values("i8")) == list(range(-127, 128))


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
def test_scale_exponent(fmt):
    top = o_kv8.code_values(fmt)[-1]
    assert o_kv8.scale_exponent(top, fmt) == 0 and o_kv8.scale_exponent(np.nextafter(top, 1e9), fmt) == 1
    assert o_kv8.scale_exponent(top / 2, fmt) == -1
    assert o_kv8.scale_exponent(0.0, fmt) == -60 and o_kv8.scale_exponent(1e38, fmt) == 60


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
def test_stored_is_the_nearest_code(fmt):
    rng = np.random.default_rng(3)
    values = o_kv8.code_values(fmt)
    x = rng.standard_normal((20, 32)) * np.exp(rng.standard_normal((20, 1)) * 8)
    got = o_kv8.stored(x, fmt)
    for row, out in zip(x, got):
        s = 2.0 ** o_kv8.scale_exponent(np.abs(row).max(), fmt)
        for a, b in zip(row, out):
            assert b / s in values and abs(a - b) <= np.abs(values * s - a).min()
    # a value that has a code is held as it is; midpoints go to the even code
    held = np.concatenate([values[:32] if fmt == "e4m3" else values[:31], [values[-1]]])
    assert (o_kv8.stored(held[None], fmt) == held).all()
    mid = (values[1:] + values[:-1]) / 2
    row = np.concatenate([mid, [values[-1]]])
    n = np.arange(len(mid)) - len(values) // 2  # number of the lower code
    assert (o_kv8.stored(row[None], fmt)[0][:-1] == np.where(n % 2 == 0, values[:-1], values[1:])).all()
    assert np.isnan(o_kv8.stored(np.array([[1.0, np.inf], [np.nan, 0.0]]), fmt)).all()
    assert (o_kv8.stored(np.zeros((1, 4)), fmt) == 0).all()


def test_attention_and_masks():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((3, 4, 32)), rng.standard_normal((9, 2, 32)), rng.standard_normal((9, 2, 32))
    everything = np.ones((3, 9), dtype=bool)
    np.testing.assert_allclose(o_kv8.attention(q, k, v, everything), o_fwd.attention(q, k, v), rtol=1e-12)
    see = everything.copy()
    see[0] = False
    see[1] = np.arange(9) == 5
    out = o_kv8.attention(q, k, v, see)
    assert (out[0] == 0).all() and np.allclose(out[1], v[5].repeat(2, axis=0))
    bad = v.copy()
    bad[2] = np.nan
    out = o_kv8.attention(q, k, bad, see)
    assert np.isfinite(out[:2]).all() and np.isnan(out[2]).all()
    # ancestors and their bits
    see = o_kv8.ancestors([-1, 0, 0, 2, -1, 3])
    assert [list(np.flatnonzero(r)) for r in see] == [[0], [0, 1], [0, 2], [0, 2, 3], [4], [0, 2, 3, 5]]
    assert o_kv8.mask_words(see, 2).tolist() == [[1, 0], [3, 0], [5, 0], [13, 0], [16, 0], [45, 0]]
    wide = np.zeros((1, 70), dtype=bool)
    wide[0, [31, 32, 69]] = True
    assert o_kv8.mask_words(wide, 3).tolist() == [[1 << 31, 1, 1 << 5]]


def test_norm_and_rotation():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 2, 32))
    y = o_kv8.qk_norm_rope(x, [0, 1, 7, 100000], np.ones(32), 1e-5, 10000.0)
    ms = (x * x).mean(-1)
    np.testing.assert_allclose((y * y).mean(-1), ms / (ms + 1e-5), rtol=1e-12)  # the rotation is an isometry
    np.testing.assert_allclose(o_kv8.qk_norm_rope(x, [0] * 4, None, 1e-5, 10000.0), x)
    a = 100000 * 10000.0 ** (-2 * 3 / 32)
    z = o_kv8.qk_norm_rope(x, [100000] * 4, None, 1e-5, 10000.0)
    np.testing.assert_allclose(z[0, 1, 3], x[0, 1, 3] * math.cos(a) - x[0, 1, 19] * math.sin(a), rtol=1e-9)
