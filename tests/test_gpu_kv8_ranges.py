"""Attention over the 8-bit cache where the scales of keys and values lie as far apart as the cache holds them.

Tolerances: those of test_gpu_kv8.py (its docstring derives them, with u, d_j, r and P), with each key's own score error instead of the largest
of all visible keys.  A probability p_j is off by p_j (e^d_j - 1) by itself and by the sum's error, which is at most a = sum_k p_k (e^d_k - 1),
so the outputs are off by sum_j p_j (e^d_j - 1) |V_j| + (a + r + (2 n + 64) u) sum_j p_j |V_j|, both times (1 + 2 a) for the second order, and by
half's end: 2^-(24+P) max_j(p_j t_j) sum_i |V_i| / t_i.  Where nothing that a row sees changes, its outputs are equal: a scale is a power of two.
"""
import math

import numpy as np
import pytest
import torch

from oracle import kv8 as o_kv8
from paper_2604_15750_amd import api
from test_gpu_kv8 import BF16, F32, HALF_STEP, U, _gen, _np64, _rows

pytestmark = pytest.mark.gpu


def _bound(q, k, v, see, dtype):
    q = _np64(q)
    n_q, hd = q.shape[1:]
    out = np.zeros(q.shape)
    for h in range(n_q):
        K, V = k[:, h * k.shape[1] // n_q], v[:, h * k.shape[1] // n_q]
        s, size = q[:, h] @ K.T / math.sqrt(hd), np.abs(q[:, h]) @ np.abs(K).T / math.sqrt(hd)
        d = ((hd + 4) * U + (2.0 ** -21 if dtype == F32 else 0.0)) * size + 8 * U * (np.abs(s) + 60 * math.log(2))
        p, t = o_kv8.probabilities(s, see), np.abs(V).max(-1, initial=0.0)
        top = np.where(see, s, -np.inf).max(-1, keepdims=True)
        log_p = np.where(see, s - top - np.log(np.exp(np.where(see, s - top, -np.inf)).sum(-1, keepdims=True)), -np.inf)
        off = np.exp(np.minimum(log_p + d, 10.0)) - np.exp(log_p)
        a = off.sum(-1, keepdims=True)
        rel = a + (2.0 ** -21 if dtype == F32 else 2.0 ** -11) + (2 * see.sum(-1, keepdims=True) + 64) * U
        end = 2.0 ** (-37 if dtype == F32 else -32) * (p * t).max(-1, initial=0.0)[:, None] * (see @ (np.abs(V) / np.maximum(t, 1e-300)[:, None]))
        out[:, h] = (1 + 2 * a) * (off @ np.abs(V) + rel * (p @ np.abs(V))) + end
    return out


def _cache(device, fmt, dtype, k, v):
    """A cache of these keys and values, and what it holds of them."""
    n, n_kv, hd = k.shape
    cache = api.Kv8Cache(1, n, n_kv, hd, fmt)
    api.dlm_kv8_write(cache, k.to(dtype).to(device), v.to(dtype).to(device), [0, n], [0])
    return cache, o_kv8.stored(_np64(k.to(dtype)), fmt), o_kv8.stored(_np64(v.to(dtype)), fmt)


def _check(device, fmt, dtype, q, k, v, see=None):
    cache, K, V = _cache(device, fmt, dtype, k, v)
    q, n, keys = q.to(dtype), len(q), len(k)
    mask = None
    if see is not None:
        mask = torch.from_numpy(o_kv8.mask_words(see, (n + 31) // 32).view(np.int32)).to(device)
    out = _np64(api.dlm_kv8_attention(cache, q.to(device), [0, n], [keys], mask=mask))
    vis = np.ones((n, keys), dtype=bool)
    if see is not None:
        vis[:, keys - n:] = see
    want = o_kv8.attention(_np64(q), K, V, vis)
    bound = _bound(q, K, V, vis, dtype) + HALF_STEP[dtype] * np.abs(want)
    assert np.isfinite(bound).all() and (bound.max(-1) < 0.5 * np.abs(V).max()).all()  # (that it says something)
    err = np.abs(out - want)
    assert (err <= bound).all(), (err / np.maximum(bound, 1e-300)).max()


CASES = [(fmt, dtype) for fmt in ("e4m3", "i8") for dtype in (BF16, F32)]


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys", [70, 3000])
@pytest.mark.parametrize("big", [2.0 ** 30, 2.0 ** 60, 3.3e38])
@pytest.mark.parametrize("q_size,k_size", [(1.0, 1.0), (2.0 ** 82, 2.0 ** -100), (2.0 ** 82, 2.0 ** -52), (2.0 ** -40, 2.0 ** 38)])
def test_finite_keys_that_a_row_does_not_see(device, fmt, dtype, keys, big, q_size, k_size):
    """Behind the keys, masked for all rows, and masked for all but one: no other row's outputs change."""
    g = _gen(keys, 41)
    n, n_kv, hd = 5, 2, 64
    k, v = _rows(g, keys + 10, n_kv, hd, F32, 0.5) * k_size, _rows(g, keys + 10, n_kv, hd, F32)
    q = (torch.randn(n, 2 * n_kv, hd, generator=g) * q_size).to(dtype).to(device)
    see = np.tril(np.ones((n, n), dtype=bool))
    see[:, 2] = False
    mask = torch.from_numpy(o_kv8.mask_words(see, 1).view(np.int32)).to(device)
    run = lambda kk: api.dlm_kv8_attention(_cache(device, fmt, dtype, kk, v)[0], q, [0, n], [keys], mask=mask)  # noqa: E731
    clean = run(k)
    assert torch.isfinite(clean).all()
    for at in (slice(keys, keys + 10), keys - n + 2, slice(keys + 3, keys + 4)):
        kk = k.clone()
        kk[at] = big * torch.sign(kk[at])
        assert torch.equal(run(kk), clean), at
    kk = k.clone()
    kk[keys - 1] = big * torch.sign(kk[keys - 1])  # (the last row sees itself)
    assert torch.equal(run(kk)[:n - 1], clean[:n - 1])


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys", [70, 3000])
@pytest.mark.parametrize("exponent", [14, 20, 26, 40, 60])
@pytest.mark.parametrize("at", [[0], [33, 64], list(range(0, 70, 3))])
def test_large_keys_without_weight(device, fmt, dtype, keys, exponent, at):
    """Keys whose scores are large and negative, in front of, among and behind the keys that have the weight."""
    g = _gen(keys, exponent, len(at))
    k, v = torch.randn(keys, 2, 64, generator=g), torch.randn(keys, 2, 64, generator=g)
    q = 0.2 + torch.rand(9, 4, 64, generator=g)
    k = k * 0.4
    k[at] = -(0.5 + torch.rand(len(at), 2, 64, generator=g)) * 2.0 ** exponent
    _check(device, fmt, dtype, q, k, v)


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys,first", [(200, 128), (200, 150), (900, 512), (3000, 1024)])
@pytest.mark.parametrize("exponent", [6, 10, 14, 17, 22, 30, 60])
def test_a_maximum_that_comes_from_far_below(device, fmt, dtype, keys, first, exponent):
    """Every wavefront's first blocks have scores of -2^8 to -2^62 (a running maximum of that size), the keys that have the weight come behind them."""
    g = _gen(keys, exponent, 7)
    k, v = torch.randn(keys, 2, 64, generator=g) * 0.4, torch.randn(keys, 2, 64, generator=g)
    q = 0.2 + torch.rand(9, 4, 64, generator=g)
    k[:first] = -(0.5 + torch.rand(first, 2, 64, generator=g)) * 2.0 ** exponent
    _check(device, fmt, dtype, q, k, v)


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys", [128, 300, 3000])
@pytest.mark.parametrize("apart", [100, 110, 120])
@pytest.mark.parametrize("where", ["first", "second block", "last"])
def test_small_values_that_have_the_weight_together(device, fmt, dtype, keys, apart, where):
    """One value, 2^apart times the others, beside keys of 2^-11 of its probability each: together they have up to one and a half times its
    weight, in its wavefront, in others and in other shares."""
    g = _gen(keys, apart)
    code = {"e4m3": 256.0, "i8": 64.0}[fmt]  # (the largest magnitude, to a scale of its own)
    at = {"first": 0, "second block": 40, "last": keys - 1}[where]
    k, v = torch.zeros(keys, 1, 64), (1 + torch.rand(keys, 1, 64, generator=g)) * code * 0.4
    v[..., 0] = code
    v = v * 2.0 ** -60
    v[at] *= 2.0 ** apart
    k[:, :, 0], k[at] = -11 * math.log(2) * 8, 0.0
    q = torch.zeros(3, 2, 64)
    q[..., 0] = 1.0
    cache, K, V = _cache(device, fmt, dtype, k, v)
    out = _np64(api.dlm_kv8_attention(cache, q.to(dtype).to(device), [0, 3], [keys]))
    vis = np.ones((3, keys), dtype=bool)
    want = o_kv8.attention(_np64(q), K, V, vis)
    assert (np.abs(out - want) <= _bound(q, K, V, vis, dtype) + HALF_STEP[dtype] * np.abs(want)).all()


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys", [70, 3000])
@pytest.mark.parametrize("exponent", [14, 26, 60])
def test_large_keys_at_right_angles(device, fmt, dtype, keys, exponent):
    """Keys that are large where the queries are zero have scores, and weights, like the others."""
    g = _gen(keys, exponent, 3)
    k, v = torch.randn(keys, 2, 64, generator=g), torch.randn(keys, 2, 64, generator=g)
    q = torch.randn(9, 4, 64, generator=g)
    q[..., :8] = 0.0
    k[5::9] = 0.0
    k[5::9, :, :8] = 2.0 ** exponent
    _check(device, fmt, dtype, q, k, v)


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys", [31, 100, 3000])
def test_keys_of_all_sizes(device, fmt, dtype, keys):
    """From 2^-56 to 2^56 in every block of 32, zeros among them; the large ones' scores are negative.  Some rows do not see some of the last positions."""
    g = _gen(keys, 5)
    rng = np.random.default_rng(keys)
    n = 20
    size = torch.exp2(torch.randint(-56, 57, (keys, 2, 1), generator=g).float())
    k = torch.randn(keys, 2, 64, generator=g)
    k = torch.where(size > 1, -k.abs(), k) * size
    k[::11] = 0.0
    k[3::4] = torch.randn(len(k[3::4]), 2, 64, generator=g) * 0.5
    v = torch.randn(keys, 2, 64, generator=g)
    q = 0.1 + torch.rand(n, 2, 64, generator=g)
    see = rng.random((n, n)) < 0.7
    _check(device, fmt, dtype, q, k, v)
    _check(device, fmt, dtype, q, k, v, see)


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys,at", [(3, 1), (70, 0), (70, 69), (3000, 2), (3000, 1777)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size(device, fmt, dtype, keys, at, sign):
    """One key's score is twice the others' (half of them, where they are negative), from 2^20 to 2^100: the output is its value."""
    g = _gen(keys, at)
    v = torch.randn(keys, 1, 64, generator=g)
    k = torch.full((keys, 1, 64), 0.5 if sign > 0 else -1.0)
    k[at] = 1.0 if sign > 0 else -0.5
    cache, _, V = _cache(device, fmt, dtype, k, v)
    q = torch.exp2(torch.tensor([*range(17, 33), 45, 60, 77, 96]).float())[:, None, None].expand(-1, 2, 64).contiguous().to(dtype)
    out = _np64(api.dlm_kv8_attention(cache, q.to(device), [0, len(q)], [keys]))
    assert (np.abs(out - V[at]) <= (HALF_STEP[dtype] + 64 * U) * np.abs(V[at])).all()


@pytest.mark.parametrize("fmt,dtype", CASES)
@pytest.mark.parametrize("keys", [300, 3000])
@pytest.mark.parametrize("value", [-60, 0, 60])
def test_large_scores_next_to_each_other(device, fmt, dtype, keys, value):
    """Scores of 2^20 to 2^60 that differ by no more than their own digits tell: any of the keys may have the weight, and all have one value."""
    g = _gen(keys, value + 100)
    k = torch.randn(keys, 1, 64, generator=g)
    k[..., 0] = 4.0
    v = torch.full((keys, 1, 64), {"e4m3": 256.0, "i8": 64.0}[fmt] * 2.0 ** value)
    q = torch.randn(20, 2, 64, generator=g)
    size = torch.exp2(torch.arange(20, 60, 2).float())[:, None]
    q[..., 0] = size
    q[..., 1:] *= 2.0 ** -20 * size[..., None]
    cache, _, V = _cache(device, fmt, dtype, k, v)
    out = _np64(api.dlm_kv8_attention(cache, q.to(dtype).to(device), [0, 20], [keys]))
    assert (np.abs(out - V[0, 0, 0]) <= (HALF_STEP[dtype] + (2 * keys + 64) * U) * V[0, 0, 0]).all()


@pytest.mark.parametrize("fmt,dtype", CASES)
def test_positions_never_written_behind_a_key_that_another_row_sees(device, fmt, dtype):
    """Queries beside whose size that key's scale has no place in 32 bits."""
    g = _gen(17)
    k, v = torch.zeros(300, 1, 32), torch.zeros(300, 1, 32)
    cache = api.Kv8Cache(1, 300, 1, 32, fmt)
    k[:20], v[:20] = torch.randn(20, 1, 32, generator=g) * 2.0 ** -84, torch.randn(20, 1, 32, generator=g)
    k[298:], v[298:] = k[:2], v[:2]
    k[298] = 2.0 ** 60
    for lo, hi in ((0, 20), (298, 300)):
        api.dlm_kv8_write(cache, k[lo:hi].to(dtype).to(device), v[lo:hi].to(dtype).to(device), [0, hi - lo], [lo])
    q = torch.ones(2, 2, 32)
    q[1] = torch.randn(2, 32, generator=g) * 2.0 ** 84
    see = np.eye(2, dtype=bool)
    mask = torch.from_numpy(o_kv8.mask_words(see, 1).view(np.int32)).to(device)
    out = _np64(api.dlm_kv8_attention(cache, q.to(dtype).to(device), [0, 2], [300], mask=mask))[1:]
    K, V = (o_kv8.stored(_np64(x.to(dtype)), fmt) for x in (k, v))
    vis = np.ones((1, 300), dtype=bool)
    vis[:, 298] = False
    want = o_kv8.attention(_np64(q[1:].to(dtype)), K, V, vis)
    bound = _bound(q[1:].to(dtype), K, V, vis, dtype) + HALF_STEP[dtype] * np.abs(want) + (2.0 ** -52 if fmt == "i8" else 0.0)
    assert (np.abs(out - want) <= bound).all()


@pytest.mark.parametrize("fmt,dtype", CASES)
def test_a_large_key_that_has_the_weight(device, fmt, dtype):
    """One row's key of 2^40: that row's output is its value; the other rows of the tile go on as they were."""
    g = _gen(8)
    n, keys = 6, 200
    k, v = torch.randn(keys, 1, 32, generator=g), torch.randn(keys, 1, 32, generator=g)
    q = 0.5 + torch.rand(n, 2, 32, generator=g)
    see = np.eye(n, dtype=bool)
    mask = torch.from_numpy(o_kv8.mask_words(see, 1).view(np.int32)).to(device)
    args = (q.to(dtype).to(device), [0, n], [keys])
    clean = api.dlm_kv8_attention(_cache(device, fmt, dtype, k, v)[0], *args, mask=mask)
    k[keys - n] = 2.0 ** 40
    cache, _, V = _cache(device, fmt, dtype, k, v)
    out = api.dlm_kv8_attention(cache, *args, mask=mask)
    assert torch.equal(out[1:], clean[1:])
    assert (np.abs(_np64(out[0]) - V[keys - n]) <= (HALF_STEP[dtype] + 64 * U) * np.abs(V[keys - n])).all()
