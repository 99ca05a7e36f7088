"""Oracle: linear layers in 8-bit integers.

TEST INFRASTRUCTURE (see oracle/__init__.py).  fp64 and whole numbers throughout.
"""
import numpy as np

from .forward import widen


def quantise(t):
    """Codes (int64) and scales (fp64) of rows t [rows, width] of fp32 values: 127 t / max|t| to the nearest, ties to even.  The quotient in fp64
    is on the right side of every border: it is off by 2^-53 of itself, and a quotient of such numbers that is no border is 2^-34 from one."""
    t = widen(t)
    top = np.abs(t).max(1, keepdims=True)
    bad = ~np.isfinite(top)
    safe = np.where(bad | (top == 0), 1.0, top)
    q = np.rint(127.0 * np.where(bad, 0.0, t) / safe).astype(np.int64)
    return q, np.where(bad, np.nan, top / 127)[:, 0]


def add_norm(x, gain, residual, eps, h_round):
    """(codes, scales, h) of dlm_add_norm_q8; h_round: what rounds a sum to the type that h has (fp64 -> fp64)."""
    x, gain = widen(x), widen(gain)
    with np.errstate(all="ignore"):
        h = x if residual is None else h_round((widen(residual) + x).astype(np.float32))
        t = (h * gain).astype(np.float32).astype(np.float64)
        q, s = quantise(t)
        return q, s / np.sqrt((h * h).mean(1) + eps), h


def product(q, s, codes, scale):
    """s_m w_n sum_k q[m][k] c[n][k], the sum in whole numbers."""
    return (q.astype(np.int64) @ codes.astype(np.int64).T).astype(np.float64) * widen(s)[:, None] * widen(scale)


def gated(y):
    """[rows, 2f] -> [rows, f]: silu of the gate times up."""
    f = y.shape[1] // 2
    g, u = y[:, :f], y[:, f:]
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-g)) * u
