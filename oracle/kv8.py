"""Oracle: the 8-bit KV cache, the norm and rotation in front of it and the attention over it.

TEST INFRASTRUCTURE (see oracle/__init__.py).  fp64 throughout, one loop or table per definition.
"""
import math

import numpy as np

from .forward import rmsnorm, rope, widen


def code_values(fmt):
    """All finite values that codes of the format stand for, ascending."""
    if fmt == "i8":
        return np.arange(-127, 128, dtype=np.float64)
    pos = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]
    return np.array(sorted(set(pos + [-p for p in pos])))


def scale_exponent(top, fmt):
    """Smallest E in [-60, 60] with top <= M 2^E (60 if there is none), for each of `top`."""
    return -60 + (np.asarray(top, dtype=np.float64)[..., None] > code_values(fmt)[-1] * 2.0 ** np.arange(-60, 60)).sum(-1)


def stored(x, fmt):
    """What vectors x [..., hd] are held as: the nearest code on each vector's scale, ties to the code with an even last bit."""
    x, values = widen(x), code_values(fmt)
    zero = len(values) // 2  # code number 0; numbers count up from it, so an even number has an even last bit
    top = np.abs(x).max(-1, keepdims=True)
    bad = ~np.isfinite(top)
    scale = 2.0 ** scale_exponent(np.where(bad, 0.0, top), fmt)
    y = np.where(bad, 0.0, x) / scale
    hi = np.clip(np.searchsorted(values, y), 1, len(values) - 1)
    lo = hi - 1
    dl, dh = y - values[lo], values[hi] - y  # (exact: y and the codes are binary fractions of few bits next to each other)
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where((lo - zero) % 2 == 0, lo, hi)))
    return np.where(bad, np.nan, values[pick] * scale)


def qk_norm_rope(x, pos, gain, eps, theta):
    """x [rows, heads, hd]; gain [hd] or None."""
    x = widen(x)
    return rope(x if gain is None else rmsnorm(x, gain, eps), pos, theta)


def probabilities(s, see):
    """softmax of scores s [A, T] over the keys that each row sees; rows that see none: zeros."""
    s = np.where(see, s, -np.inf)
    p = np.exp(s - np.where(see.any(-1, keepdims=True), s.max(-1, keepdims=True, initial=-np.inf), 0.0))
    return p / np.maximum(p.sum(-1, keepdims=True), 1e-300)


def attention(q, k, v, see):
    """q [A, n_q, hd], k and v [T, n_kv, hd]; see [A, T]: which keys a row attends to.  Rows without any: zeros; rows that see a key or
    value with a NaN: NaN."""
    q, k, v = widen(q), widen(k), widen(v)
    n_q, hd = q.shape[1:]
    out = np.empty(q.shape)
    for h in range(n_q):
        K, V = k[:, h * k.shape[1] // n_q], v[:, h * k.shape[1] // n_q]
        bad = np.isnan(K).any(-1) | np.isnan(V).any(-1)
        s = q[:, h] @ np.where(bad[:, None], 0.0, K).T / math.sqrt(hd)
        out[:, h] = probabilities(s, see) @ np.where(bad[:, None], 0.0, V)
        out[(see & bad).any(-1), h] = np.nan
    return out


def ancestors(parent):
    """see [n, n] of a tree of drafted tokens: a node sees itself and its ancestors (parent[i] < i, -1: a root)."""
    n = len(parent)
    see = np.zeros((n, n), dtype=bool)
    for i in range(n):
        j = i
        while j >= 0:
            see[i, j] = True
            j = parent[j]
    return see


def mask_words(see, words):
    """Bit j % 32 of word j / 32 of a row: it sees position j."""
    out = np.zeros((see.shape[0], words), dtype=np.uint32)
    for r, j in zip(*np.nonzero(see)):
        out[r, j // 32] |= np.uint32(1 << (j % 32))
    return out
