"""The 8-bit cache's operators on the GPU against the 64-bit oracle (oracle/kv8.py).

Tolerances, derived before the first run (u = 2^-24, half a step of fp32; a rounding to bf16 is off by at most 2^-8 of the value):
  write / read   none: a scale is a power of two, so a code depends on the vector alone; bf16 and fp32 hold every cached value exactly
  norm + rope    fp32 up to the output: the sum of squares, its root and two products (<= 16 u of the normalised value), the angle's
                 cosine and sine (<= 4 u each) and the two products' sum: 32 u of |y_i| + |y_j|, then the output's rounding
  attention      scores: hd + 4 roundings of partial sums no larger than sum_i |q_i K_ji| (fp32 queries: and 2^-21 of each q), and 8
                 roundings of a log2 score plus V's exponent: d_j = (hd + 4) u sum|q_i K_ji| / sqrt(hd) + 8 u (|s_j| + 60 ln 2); a
                 probability is off by 2 d of itself (its own and the sum's) and by its rounding to half (2^-11 bf16, two terms 2^-21
                 fp32); sums over n keys 2 n u.  So (2 max d + r + (2 n + 64) u) sum_j p_j |V_j|, then the output's rounding.  Half ends:
                 what multiplies the codes is p_j 2^b_j (b: the exponent of V_j's scale) with its largest at 2^P or above (P = 8 with bf16,
                 13 with fp32 outputs), and below 2^-14 half's steps are 2^-24, so each is off by up to 2^-25 = 2^-(25+P) of the
                 largest: 2^-(25+P) max_j(p_j 2^b_j) sum_i |code_i|.  With t the largest magnitude of a vector and M the largest code,
                 2^b <= 2 t / M and |code| <= M |V| / t: at most 2^-(24+P) max_j(p_j t_j) sum_i |V_i| / t_i
"""
import math

import numpy as np
import pytest
import torch

from oracle import kv8 as o_kv8
from paper_2604_15750_amd import api, inputs

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, F32: U}


def _np64(t):
    return t.detach().cpu().double().numpy()


def _gen(*key):
    return torch.Generator(device="cpu").manual_seed(sum(k * 7919 ** i for i, k in enumerate(key)) % (1 << 62))


def _rows(g, n, n_kv, hd, dtype, spread=2.0):
    """Vectors of widely different magnitudes."""
    return (torch.randn(n, n_kv, hd, generator=g) * torch.exp(spread * torch.randn(n, n_kv, 1, generator=g))).to(dtype)


def _strided(x, device, gap=8):
    """x on the device as columns of a wider matrix."""
    rows = x.reshape(x.shape[0], -1)
    wide = torch.full((rows.shape[0], rows.shape[1] + 2 * gap), 3.0, dtype=x.dtype)
    wide[:, gap:gap + rows.shape[1]] = rows
    return wide.to(device)[:, gap:gap + rows.shape[1]].unflatten(1, x.shape[1:])


# ---- the cache -------------------------------------------------------------------------------------------------------------------

SPANS = [  # (max_len, [(slot, first position, rows)])
    (1, [(0, 0, 1)]),
    (32, [(0, 31, 1)]),
    (70, [(1, 0, 70), (0, 5, 1)]),
    (200, [(2, 33, 100), (0, 0, 32), (3, 31, 2), (1, 64, 0), (4, 17, 64)]),
    (333, [(0, 1, 332)]),
]


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n_kv", [(32, 3), (64, 2), (128, 5)])
@pytest.mark.parametrize("max_len,spans", SPANS)
def test_written_spans_read_back(device, fmt, dtype, hd, n_kv, max_len, spans):
    g = _gen(hd, max_len, len(spans))
    cache = api.Kv8Cache(5, max_len, n_kv, hd, fmt)
    # every position first holds something else, so that a write outside its span shows
    old = [_rows(g, 5 * max_len, n_kv, hd, dtype) for _ in "kv"]
    api.dlm_kv8_write(cache, *(x.to(device) for x in old), [i * max_len for i in range(6)], [0] * 5)
    off = [0]
    for _, _, n in spans:
        off.append(off[-1] + n)
    new = [_rows(g, off[-1] + 3, n_kv, hd, dtype) for _ in "kv"]
    start, slot = [s[1] for s in spans], [s[0] for s in spans]
    api.dlm_kv8_write(cache, *(_strided(x, device) for x in new), off, start, slot)
    want = [o_kv8.stored(_np64(x), fmt).reshape(5, max_len, n_kv, hd) for x in old]
    for i in range(2):
        held = o_kv8.stored(_np64(new[i]), fmt)
        for b, (s, first, n) in enumerate(spans):
            want[i][s, first:first + n] = held[off[b]:off[b + 1]]
    got = api.dlm_kv8_read(cache, [i * max_len for i in range(6)], [0] * 5, dtype=dtype)
    # the spans alone, into rows of a wider matrix with rows behind the last sequence
    part = [_strided(torch.full((off[-1] + 2, n_kv, hd), 9.0, dtype=dtype), device) for _ in "kv"]
    api.dlm_kv8_read(cache, off, start, slot, k=part[0], v=part[1])
    torch.cuda.synchronize()
    for i in range(2):
        assert (_np64(got[i]).reshape(want[i].shape) == want[i]).all()
        for b, (s, first, n) in enumerate(spans):
            assert (_np64(part[i])[off[b]:off[b + 1]] == want[i][s, first:first + n]).all()
        assert (part[i][off[-1]:] == 9).all() and (part[i]._base[:, [0, -1]] == 3).all()


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_codes_at_their_borders(device, fmt, dtype):
    """Every code, every midpoint of two and its neighbours, on scales from the smallest to the largest; saturation behind both ends."""
    values = o_kv8.code_values(fmt)
    mid = (values[1:] + values[:-1]) / 2
    eps = float(torch.finfo(dtype).eps)
    row = np.concatenate([values, mid, mid * (1 + eps), mid * (1 - eps), [2.0 ** -12, 2.0 ** -10 * (1 + eps)]])
    row = np.concatenate([row, np.zeros(-len(row) % 31)]).reshape(-1, 31)
    row = np.concatenate([row, np.full((len(row), 1), values[-1])], 1)  # each vector's largest: scale 2^0
    x = np.concatenate([row * 2.0 ** e for e in (-100, -61, -60, -59, 0, 13, 59, 60, 61, 100)])
    x = torch.from_numpy(x).to(dtype)[:, None]
    cache = api.Kv8Cache(1, len(x), 1, 32, fmt)
    api.dlm_kv8_write(cache, x.to(device), (-x).contiguous().to(device), [0, len(x)], [0])
    k, v = api.dlm_kv8_read(cache, [0, len(x)], [0], dtype=dtype)
    want = o_kv8.stored(_np64(x), fmt)
    assert (_np64(k) == want).all() and (_np64(v) == -want).all()


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
def test_vectors_with_nan_or_infinity_and_positions_never_written(device, fmt):
    g = _gen(9)
    x = _rows(g, 40, 2, 64, F32)
    k, v = x.clone(), x.flip(0).clone()
    k[3, 1, 5], k[4, 0, 63], v[7, 1, 0], k[6] = math.nan, math.inf, -math.inf, 0.0
    cache = api.Kv8Cache(1, 64, 2, 64, fmt)
    api.dlm_kv8_write(cache, k.to(device), v.to(device), [0, 40], [8])
    got = api.dlm_kv8_read(cache, [0, 64], [0], dtype=F32)
    for x, y in zip((k, v), got):
        y = _np64(y)
        assert np.array_equal(y[8:48], o_kv8.stored(_np64(x), fmt), equal_nan=True)
        assert (y[:8] == 0).all() and (y[48:] == 0).all()


# ---- norm and rotation -------------------------------------------------------------------------------------------------------------

def _norm_rope_reference(x, pos, n_q, n_kv, hd, gq, gk, eps, theta):
    heads = _np64(x)[:, :(n_q + n_kv) * hd].reshape(-1, n_q + n_kv, hd)
    out, size = [], []
    for lo, n, gain in ((0, n_q, gq), (n_q, n_kv, gk)):
        g = None if gain is None else _np64(gain)
        y = o_kv8.qk_norm_rope(heads[:, lo:lo + n], [0] * len(heads), g, eps, theta)
        out.append(o_kv8.qk_norm_rope(heads[:, lo:lo + n], _np64(pos), g, eps, theta))
        y = np.abs(y)
        size.append(y + np.roll(y, hd // 2, -1))
    return np.concatenate(out, 1), np.concatenate(size, 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n_q,n_kv", [(32, 4, 4), (64, 16, 2), (128, 28, 4), (128, 1, 0), (64, 0, 3), (32, 33, 1), (128, 71, 2)])
@pytest.mark.parametrize("rows", [1, 5, 64])
def test_qk_norm_rope(device, dtype, hd, n_q, n_kv, rows):
    g = _gen(hd, n_q, rows)
    width = (n_q + n_kv) * hd
    x = _rows(g, rows, 1, width + 64, dtype)[:, 0]
    pos = torch.randint(-1000, 1 << 20, (rows,), generator=g, dtype=torch.int32)
    pos[0] = 0
    if rows > 2:
        pos[1], pos[2] = 2 ** 31 - 1, -2 ** 31
    gq, gk = ((1 + 0.3 * torch.randn(hd, generator=g)).to(dtype) for _ in "qk")
    for gains, theta in (((gq, gk), 10000.0), ((None, gk), 1e6), ((gq, None), 500.0)):
        dev = [None if t is None else t.to(device) for t in gains]
        xd = x.to(device)
        got = api.dlm_qk_norm_rope(xd, pos.to(device), n_q, n_kv, hd, *dev, eps=1e-5, theta=theta)
        want, size = _norm_rope_reference(x, pos, n_q, n_kv, hd, *gains, 1e-5, theta)
        got64 = _np64(got).reshape(want.shape)
        bound = HALF_STEP[dtype] * np.abs(want) + 32 * U * (1 + HALF_STEP[dtype]) * size
        assert (np.abs(got64 - want) <= bound).all(), (np.abs(got64 - want) / np.maximum(bound, 1e-300)).max()
        # in place: the same values, and what lies behind the heads stays
        api.dlm_qk_norm_rope(xd, pos.to(device), n_q, n_kv, hd, *dev, eps=1e-5, theta=theta, out=xd)
        assert torch.equal(xd[:, :width], got) and torch.equal(xd[:, width:].cpu(), x[:, width:])


# ---- attention -----------------------------------------------------------------------------------------------------------------------

def _bound(q, k, v, see, dtype):
    """Per output: what the docstring above derives."""
    q = _np64(q)
    n_q, hd = q.shape[1:]
    out = np.zeros(q.shape)
    seen = see.sum(-1)
    for h in range(n_q):
        K, V = k[:, h * k.shape[1] // n_q], v[:, h * k.shape[1] // n_q]
        s, size = q[:, h] @ K.T / math.sqrt(hd), np.abs(q[:, h]) @ np.abs(K).T / math.sqrt(hd)
        d = ((hd + 4) * U + (2.0 ** -21 if dtype == F32 else 0.0)) * size + 8 * U * (np.abs(s) + 60 * math.log(2))
        rel = 2 * np.where(see, d, 0.0).max(-1, initial=0.0) + (2.0 ** -21 if dtype == F32 else 2.0 ** -11) + (2 * seen + 64) * U
        p, t = o_kv8.probabilities(s, see), np.abs(V).max(-1, initial=0.0)
        out[:, h] = rel[:, None] * (p @ np.abs(V)) + 2.0 ** (-37 if dtype == F32 else -32) * (p * t).max(-1, initial=0.0)[:, None] * (see @ (np.abs(V) / np.maximum(t, 1e-300)[:, None]))
    return out


def _run(device, fmt, dtype, n_q, n_kv, hd, seqs, see=None, words=None, q_scale=1.0, spread=0.7, key=0, junk_bits=False):
    """seqs: (slot, rows, keys).  see: per sequence [rows, rows] or None.  Checks the attention over a cache that holds more than the
    keys; returns what the caller may compare."""
    g = _gen(n_q, hd, key, len(seqs))
    slots = max(s[0] for s in seqs) + 1
    longest = max(s[2] for s in seqs)
    max_len = longest + 37
    cache = api.Kv8Cache(slots, max_len, n_kv, hd, fmt)
    kv = [_rows(g, slots * max_len, n_kv, hd, dtype, spread) for _ in "kv"]
    api.dlm_kv8_write(cache, *(x.to(device) for x in kv), [i * max_len for i in range(slots + 1)], [0] * slots)
    K, V = (o_kv8.stored(_np64(x), fmt).reshape(slots, max_len, n_kv, hd) for x in kv)
    off = [0]
    for _, n, _ in seqs:
        off.append(off[-1] + n)
    q = (torch.randn(off[-1] + 1, n_q, hd, generator=g) * q_scale).to(dtype)
    mask = None
    if see is not None:
        words = words or max(1, (max(s[1] for s in seqs) + 31) // 32)
        bits = np.zeros((off[-1] + 1, words), dtype=np.uint32)
        for b, s in enumerate(see):
            bits[off[b]:off[b + 1]] = o_kv8.mask_words(s, words)
            if junk_bits:  # bits that stand for no row
                for j in range(s.shape[1], 32 * words):
                    bits[off[b]:off[b + 1], j // 32] |= np.uint32(1 << (j % 32))
        mask = torch.from_numpy(bits.view(np.int32)).to(device)
    out = torch.full((off[-1] + 1, n_q, hd), 5.0, dtype=dtype, device=device)
    qd = _strided(q, device)
    args = (cache, qd, off, [s[2] for s in seqs], [s[0] for s in seqs], mask)
    api.dlm_kv8_attention(*args, out=out)
    again = api.dlm_kv8_attention(*args)
    assert torch.equal(again[:off[-1]], out[:off[-1]]) and (out[off[-1]:] == 5).all()
    for b, (slot, n, keys) in enumerate(seqs):
        if n == 0:
            continue
        vis = np.ones((n, keys), dtype=bool)
        if see is not None:
            vis[:, keys - n:] = see[b]
        rows = slice(off[b], off[b + 1])
        want = o_kv8.attention(_np64(q[rows]), K[slot, :keys], V[slot, :keys], vis)
        bound = _bound(q[rows], K[slot, :keys], V[slot, :keys], vis, dtype) + HALF_STEP[dtype] * np.abs(want)
        err = np.abs(_np64(out[rows]) - want)
        assert (err <= bound).all(), (b, (err / np.maximum(bound, 1e-300)).max())
    return cache, q, out, K, V


HEADS = [(4, 4, 32), (16, 2, 64), (7, 1, 128), (3, 3, 128)]
SEQS = [
    [(0, 1, 1)],
    [(0, 1, 0), (1, 2, 31), (2, 0, 5), (3, 3, 33)],         # no keys, no rows, odd lengths
    [(1, 8, 64), (0, 17, 129), (1, 1, 40)],                 # a slot twice
    [(0, 40, 100)],
    [(0, 1, 3001), (1, 2, 200)],                            # keys split over workgroups, a short sequence beside a long one
]


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_q,n_kv,hd", HEADS)
@pytest.mark.parametrize("seqs", SEQS)
def test_attention(device, fmt, dtype, n_q, n_kv, hd, seqs):
    _run(device, fmt, dtype, n_q, n_kv, hd, seqs)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_many_rows(device, dtype):
    """Several query tiles a workgroup, ragged at the end, more workgroups than the chip takes at once."""
    _run(device, "e4m3", dtype, 2, 2, 64, [(0, 131, 300), (1, 200, 200)])
    _run(device, "i8", dtype, 70, 70, 32, [(0, 70, 70), (1, 65, 97), (2, 33, 64), (3, 64, 64)])


def _trees(seqs, seed):
    rng = np.random.default_rng(seed)
    return [o_kv8.ancestors([int(rng.integers(max(-1, i - 6), i)) for i in range(n)]) for _, n, _ in seqs]


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_q,n_kv,hd", [(4, 4, 32), (7, 1, 128)])
@pytest.mark.parametrize("seqs", [[(0, 1, 1)], [(0, 12, 12), (1, 5, 40)], [(0, 33, 70), (1, 64, 64), (2, 7, 1500)], [(0, 70, 101)]])
def test_attention_of_trees(device, fmt, dtype, n_q, n_kv, hd, seqs):
    _run(device, fmt, dtype, n_q, n_kv, hd, seqs, see=_trees(seqs, 5))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masks_of_any_kind(device, dtype):
    """Rows that see nothing, everything, one position, those behind themselves; words and bits that stand for no row; every alignment of the
    masked positions to the blocks of 32."""
    rng = np.random.default_rng(6)
    for keys, n in [(n + p, n) for n in (1, 31, 32, 33, 45) for p in (0, 1, 19, 31, 32, 50)]:
        see = rng.random((n, n)) < 0.4
        see[0] = False
        see[n // 2] = True
        see[-1] = np.arange(n) == n - 1 if n > 1 else False
        _run(device, "e4m3", dtype, 2, 1, 32, [(0, n, keys)], see=[see], words=3, key=keys, junk_bits=True)
    out = _run(device, "i8", dtype, 2, 2, 32, [(0, 3, 3)], see=[np.zeros((3, 3), dtype=bool)])[2]
    assert (out[:3] == 0).all()


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scales_far_apart(device, fmt, dtype):
    """Values, keys and queries of magnitudes from 2^-50 to 2^50 in one softmax: every probability keeps its weight whatever its value's scale."""
    _run(device, fmt, dtype, 2, 2, 64, [(0, 20, 150), (1, 3, 700)], spread=6.0, key=1, q_scale=1e-3)
    g = _gen(3)
    cache = api.Kv8Cache(1, 128, 1, 64, fmt)
    k = torch.randn(128, 1, 64, generator=g)
    v = torch.randn(128, 1, 64, generator=g) * torch.exp2(torch.randint(-50, 51, (128, 1, 1), generator=g).float())
    k, v = k.to(dtype), v.to(dtype)
    api.dlm_kv8_write(cache, k.to(device), v.to(device), [0, 128], [0])
    K, V = (o_kv8.stored(_np64(x), fmt) for x in (k, v))
    q = torch.randn(40, 1, 64, generator=g) * torch.exp2(torch.randint(-60, 3, (40, 1, 1), generator=g).float())
    q[7], q[8] = 0.0, q[8] * 2.0 ** 20
    q = q.to(dtype)
    out = api.dlm_kv8_attention(cache, q.to(device), [0, 40], [128])
    see = np.ones((40, 128), dtype=bool)
    want = o_kv8.attention(_np64(q), K, V, see)
    bound = _bound(q, K, V, see, dtype) + HALF_STEP[dtype] * np.abs(want)
    err = np.abs(_np64(out) - want)
    assert (err <= bound).all(), (err / bound).max()
    # a value of 2^-50 that has all the weight, beside one of 2^50 that has none
    k = torch.zeros(2, 1, 32)
    k[0], k[1] = 4.0, -4.0
    v = torch.stack([torch.full((1, 32), 2.0 ** -50), torch.full((1, 32), 2.0 ** 50)])
    cache = api.Kv8Cache(1, 2, 1, 32, fmt)
    api.dlm_kv8_write(cache, k.to(dtype).to(device), v.to(dtype).to(device), [0, 2], [0])
    q = torch.full((1, 1, 32), 8.0, dtype=dtype)
    out = _np64(api.dlm_kv8_attention(cache, q.to(device), [0, 1], [2]))
    want = o_kv8.attention(_np64(q), _np64(k), _np64(v), np.ones((1, 2), dtype=bool))
    assert (np.abs(out - want) <= (2 * HALF_STEP[dtype] + 1e-4) * np.abs(want)).all()  # one key has all the weight: p = 1


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("big", [False, True])
def test_attention_sees_positions_never_written(device, fmt, dtype, big):
    """They are keys and values of zeros, whichever wavefront or share has them and whatever the scales of the others.  (i8: the code is
    -128 at 2^-60, so up to 2^-53 for zero.)"""
    g = _gen(31, big)
    for keys, spans in ((64, [(0, 32)]), (290, [(3, 40), (200, 20)]), (3000, [(1500, 300)]), (40, [])):
        k, v = torch.zeros(keys, 2, 64), torch.zeros(keys, 2, 64)
        cache = api.Kv8Cache(1, keys, 2, 64, fmt)
        for at, n in spans:
            k[at:at + n] = torch.randn(n, 2, 64, generator=g)
            v[at:at + n] = torch.randn(n, 2, 64, generator=g) * (2.0 ** 45 if big else 1.0)
            api.dlm_kv8_write(cache, k[at:at + n].to(dtype).to(device), v[at:at + n].to(dtype).to(device), [0, n], [at])
        K, V = (o_kv8.stored(_np64(x.to(dtype)), fmt) for x in (k, v))
        q = torch.randn(5, 4, 64, generator=g).to(dtype)
        see = np.ones((5, keys), dtype=bool)
        want = o_kv8.attention(_np64(q), K, V, see)
        bound = _bound(q, K, V, see, dtype) + HALF_STEP[dtype] * np.abs(want) + (2.0 ** -52 if fmt == "i8" else 0.0)
        err = np.abs(_np64(api.dlm_kv8_attention(cache, q.to(device), [0, 5], [keys])) - want)
        assert (err <= bound).all(), (keys, (err / np.maximum(bound, 1e-300)).max())


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("keys", [70, 3000])
def test_nan_and_infinity(device, fmt, dtype, keys):
    """In places that a row does not see they change nothing; what a row sees makes that row (and head) NaN, and no other."""
    g = _gen(keys)
    n, n_kv, hd = 5, 2, 64
    k, v = _rows(g, keys + 10, n_kv, hd, dtype), _rows(g, keys + 10, n_kv, hd, dtype)
    q = torch.randn(n, 2 * n_kv, hd, generator=g).to(dtype)
    see = np.tril(np.ones((n, n), dtype=bool))
    see[:, 2] = False
    see[4, 3] = False
    mask = torch.from_numpy(o_kv8.mask_words(see, 1).view(np.int32)).to(device)
    clean = [x.clone() for x in (k, v)]
    k[keys - n + 2], v[keys - n + 2] = math.nan, math.inf  # seen by nobody
    k[keys:], v[keys:] = math.inf, math.nan                # behind the keys
    caches = []
    for kk, vv in (clean, (k, v)):
        caches.append(api.Kv8Cache(1, keys + 10, n_kv, hd, fmt))
        api.dlm_kv8_write(caches[-1], kk.to(device), vv.to(device), [0, keys + 10], [0])
    a, b = (api.dlm_kv8_attention(c, q.to(device), [0, n], [keys], mask=mask) for c in caches)
    assert torch.isfinite(b).all() and torch.equal(a, b)
    # position keys - 2 (row 3 sees it) in V of head 1; the first position in K of head 0
    for which, pos, head, rows in ((1, keys - 2, 1, [3]), (0, 0, 0, [0, 1, 2, 3, 4]), (0, keys - 2, 1, [3]), (1, 0, 0, [0, 1, 2, 3, 4])):
        kv = [x.clone() for x in clean]
        kv[which][pos, head, 9] = math.nan
        api.dlm_kv8_write(caches[1], *(x.to(device) for x in kv), [0, keys + 10], [0])
        b = api.dlm_kv8_attention(caches[1], q.to(device), [0, n], [keys], mask=mask).view(n, n_kv, 2, hd)
        bad = torch.zeros(n, n_kv, dtype=torch.bool)
        bad[rows, head] = True
        assert torch.equal(torch.isnan(b).all(-1).all(-1).cpu(), bad) and torch.equal(torch.isnan(b).any(-1).any(-1).cpu(), bad)
        assert torch.equal(b[~bad.to(device)], a.view(n, n_kv, 2, hd)[~bad.to(device)])
    # a query that is not finite is its own row's and head's matter
    q2 = q.clone()
    q2[1, 3, 7], q2[4, 0, 0] = math.nan, math.inf
    b = api.dlm_kv8_attention(caches[0], q2.to(device), [0, n], [keys], mask=mask)
    bad = torch.zeros(n, 2 * n_kv, dtype=torch.bool)
    bad[1, 3] = bad[4, 0] = True
    assert torch.equal(torch.isnan(b).any(-1).cpu(), bad) and torch.equal(b[~bad.to(device)], a[~bad.to(device)])


def test_cache_beyond_32_bits(device):
    """Slots whose codes lie more than 4 GiB into the cache."""
    g = _gen(11)
    slots, max_len, n_kv, hd = 36, 16400, 32, 128
    cache = api.Kv8Cache(slots, max_len, n_kv, hd, "e4m3")
    assert cache.data.numel() > 1 << 32
    x = torch.randn(16400, n_kv, hd, generator=g).to(BF16).to(device)
    api.dlm_kv8_write(cache, x[:900], x[900:1800], [0, 900], [15500], [35])
    api.dlm_kv8_write(cache, x[:300], x[300:600], [0, 300], [0], [0])
    k, v = api.dlm_kv8_read(cache, [0, 900], [15500], [35])
    small = api.Kv8Cache(1, 900, n_kv, hd, "e4m3")
    api.dlm_kv8_write(small, x[:900], x[900:1800], [0, 900], [0])
    assert all(torch.equal(a, b) for a, b in zip((k, v), api.dlm_kv8_read(small, [0, 900], [0])))
    api.dlm_kv8_write(cache, x, x, [0, 16400], [0], [35])
    q = torch.randn(2, 32, hd, generator=g).to(BF16).to(device)
    out = api.dlm_kv8_attention(cache, q, [0, 2], [16400], [35])
    k, v = (t.double() for t in api.dlm_kv8_read(cache, [0, 16400], [0], [35]))
    s = (q.double()[:, None] * k).sum(-1) / math.sqrt(hd)  # [2, keys, heads]
    p = torch.softmax(s, 1)
    want, size = (p[..., None] * v).sum(1), (p[..., None] * v.abs()).sum(1)
    # sum|q K| / sqrt(hd) of unit normals: below 40; d <= 132 u 40 + 8 u 55 = 3.5e-4; then 2^-11 and 2 n u = 2e-3
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2 * 3.5e-4 + 2.0 ** -11 + 2e-3) * size).all()


# ---- together --------------------------------------------------------------------------------------------------------------------------

def _chain(cache, qkv, positions, gains, n_q, n_kv, hd, off, start, ends, mask, ws, out):
    """A pass's attention: norm and rotation in place, the rows' K and V into the cache, the rows over it."""
    api.dlm_qk_norm_rope(qkv, positions, n_q, n_kv, hd, *gains, out=qkv)
    q, k, v = qkv.split([n_q * hd, n_kv * hd, n_kv * hd], 1)
    api.dlm_kv8_write(cache, k.unflatten(1, (n_kv, hd)), v.unflatten(1, (n_kv, hd)), off, start)
    return api.dlm_kv8_attention(cache, q.unflatten(1, (n_q, hd)), off, ends, mask=mask, workspace=ws, out=out)


def _chain_inputs(device, fmt, dtype, key):
    g = _gen(21, key)
    n_q, n_kv, hd, spans = 8, 2, 64, [(40, 9), (700, 33), (0, 5)]  # (cached, drafted)
    cache = api.Kv8Cache(3, 800, n_kv, hd, fmt)
    for b, (n, _) in enumerate(spans):
        if n:
            api.dlm_kv8_write(cache, *(_rows(g, n, n_kv, hd, dtype, 0.5).to(device) for _ in "kv"), [0, n], [0], [b])
    off = [0, 9, 42, 47]
    trees = _trees([(0, n, 0) for _, n in spans], key)
    depth = np.concatenate([[spans[b][0] + s[i].sum() - 1 for i in range(len(s))] for b, s in enumerate(trees)])
    qkv = torch.randn(47, (n_q + 2 * n_kv) * hd, generator=g).to(dtype)
    gains = [(1 + 0.2 * torch.randn(hd, generator=g)).to(dtype) for _ in "qk"]
    mask = np.concatenate([o_kv8.mask_words(s, 2) for s in trees]).view(np.int32)
    return dict(n_q=n_q, n_kv=n_kv, hd=hd, spans=spans, cache=cache, off=off, trees=trees, depth=depth, qkv=qkv, gains=gains, mask=torch.from_numpy(mask).to(device),
                positions=torch.from_numpy(depth.astype(np.int32)).to(device), start=[s[0] for s in spans], ends=[sum(s) for s in spans])


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_drafted_trees_end_to_end(device, fmt, dtype):
    c = _chain_inputs(device, fmt, dtype, 1)
    n_q, n_kv, hd, off = c["n_q"], c["n_kv"], c["hd"], c["off"]
    gains = [x.to(device) for x in c["gains"]]
    qkv = c["qkv"].to(device)
    out = _chain(c["cache"], qkv, c["positions"], gains, n_q, n_kv, hd, off, c["start"], c["ends"], c["mask"], None, None)
    # each stage on the one before it
    want, size = _norm_rope_reference(c["qkv"], torch.from_numpy(c["depth"]), n_q, n_kv, hd, *c["gains"], 1e-5, 10000.0)
    got = _np64(qkv)[:, :(n_q + n_kv) * hd].reshape(want.shape)
    assert (np.abs(got - want) <= HALF_STEP[dtype] * np.abs(want) + 32 * U * (1 + HALF_STEP[dtype]) * size).all()
    kv = api.dlm_kv8_read(c["cache"], off, c["start"], dtype=dtype)
    for x, cols in zip(kv, (slice(n_q * hd, (n_q + n_kv) * hd), slice((n_q + n_kv) * hd, None))):
        assert (_np64(x) == o_kv8.stored(_np64(qkv[:, cols]).reshape(-1, n_kv, hd), fmt)).all()
    for b, keys in enumerate(c["ends"]):
        K, V = (_np64(x) for x in api.dlm_kv8_read(c["cache"], [0, keys], [0], [b], dtype=dtype))
        rows, n = slice(off[b], off[b + 1]), off[b + 1] - off[b]
        see = np.ones((n, keys), dtype=bool)
        see[:, keys - n:] = c["trees"][b]
        q = qkv[rows, :n_q * hd].unflatten(1, (n_q, hd))
        want = o_kv8.attention(_np64(q), K, V, see)
        err = np.abs(_np64(out[rows]) - want)
        assert (err <= _bound(q, K, V, see, dtype) + HALF_STEP[dtype] * np.abs(want)).all()
    # an accepted path: its rows again, at the positions behind the prefix; attention over it equals that of its last node
    path = list(np.flatnonzero(c["trees"][1][-1]))
    rows = qkv[off[1]:off[2]][path].contiguous()
    k, v = (rows[:, cols].unflatten(1, (n_kv, hd)) for cols in (slice(n_q * hd, (n_q + n_kv) * hd), slice((n_q + n_kv) * hd, None)))
    before = out[off[2] - 1].clone()
    api.dlm_kv8_write(c["cache"], k, v, [0, len(path)], [c["start"][1]], [1])
    q = rows[-1:, :n_q * hd].unflatten(1, (n_q, hd))
    after = api.dlm_kv8_attention(c["cache"], q, [0, 1], [c["start"][1] + len(path)], [1])
    K, V = (_np64(x) for x in api.dlm_kv8_read(c["cache"], [0, c["start"][1] + len(path)], [0], [1], dtype=dtype))
    see = np.ones((1, len(K)), dtype=bool)
    twice = 2 * (_bound(q, K, V, see, dtype) + HALF_STEP[dtype] * np.abs(_np64(after[:1])))  # (two sums of the same terms in another order)
    assert (np.abs(_np64(before)[None] - _np64(after)) <= twice * 1.01).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_and_on_another_stream(device, dtype):
    """Two captured passes with a workspace each, replayed in turn and between eager work, against the eager results bit for bit."""
    cases = [_chain_inputs(device, "e4m3", dtype, 1), _chain_inputs(device, "i8", dtype, 2)]
    eager, graphs = [], []
    for c in cases:
        c["gains"] = [x.to(device) for x in c["gains"]]
        c["x"] = c["qkv"].to(device)
        c["src"] = c["x"].clone()
        need = api.lib().dlm_kv8_attention_workspace(c["off"][-1], c["n_q"], c["hd"])
        c["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
        c["out"] = torch.empty(c["off"][-1], c["n_q"], c["hd"], dtype=dtype, device=device)
        c["call"] = lambda c=c: _chain(c["cache"], c["x"], c["positions"], c["gains"], c["n_q"], c["n_kv"], c["hd"], c["off"], c["start"], c["ends"], c["mask"],
                                       c["ws"], c["out"])
        eager.append(c["call"]().clone())
    side = torch.cuda.Stream()
    for c in cases:
        c["x"].copy_(c["src"])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c["call"]()
        graphs.append(g)
    for _ in range(3):
        for i in (0, 1, 1):
            c = cases[i]
            c["x"].copy_(c["src"])
            c["out"].fill_(7)
            graphs[i].replay()
            assert torch.equal(c["out"], eager[i])
        torch.cuda.synchronize()
    # eager on a stream of its own, the other case meanwhile on the default one
    for c in cases:
        c["x"].copy_(c["src"])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        a = cases[0]["call"]().clone()
    b = cases[1]["call"]().clone()
    torch.cuda.synchronize()
    assert torch.equal(a, eager[0]) and torch.equal(b, eager[1])


def test_columns_of_one_matrix(device):
    """q, k and v read into, and heads rotated into, other columns of the matrix they come from."""
    g = _gen(21)
    wide = torch.randn(9, 5 * 128, generator=g).to(BF16).to(device)
    part = lambda i: wide[:, 128 * i:128 * (i + 1)]  # noqa: E731
    pos = torch.arange(9, dtype=torch.int32, device=device)
    want = api.dlm_qk_norm_rope(part(0).contiguous(), pos, 2, 0, 64)
    before = wide.clone()
    api.dlm_qk_norm_rope(part(0), pos, 2, 0, 64, out=part(1))
    assert torch.equal(part(1), want)
    cache = api.Kv8Cache(1, 9, 2, 64)
    heads = lambda i: part(i).unflatten(1, (2, 64))  # noqa: E731
    api.dlm_kv8_write(cache, heads(0), heads(1), [0, 9], [0])
    api.dlm_kv8_read(cache, [0, 9], [0], k=heads(4), v=heads(3))
    k, v = api.dlm_kv8_read(cache, [0, 9], [0])
    assert torch.equal(heads(4), k) and torch.equal(heads(3), v)
    assert torch.equal(part(0), before[:, :128]) and torch.equal(part(2), before[:, 256:384])


def test_empty_calls_and_refusals(device):
    cache, long = api.Kv8Cache(2, 64, 2, 64, "e4m3"), api.Kv8Cache(1, 2000, 2, 64, "e4m3")
    x = torch.randn(6, 2, 64, device=device).to(BF16)
    none = x[:0]
    api.dlm_kv8_write(cache, none, none, [0, 0], [3])
    assert api.dlm_kv8_read(cache, [0, 0], [3])[0].shape == (0, 2, 64)
    assert api.dlm_kv8_attention(cache, none, [0, 0], [3]).shape == (0, 2, 64)
    assert api.dlm_qk_norm_rope(none.flatten(1), torch.zeros(0, dtype=torch.int32, device=device), 1, 1, 64).shape == (0, 128)
    pos = torch.zeros(6, dtype=torch.int32, device=device)
    for call in (lambda: api.dlm_kv8_write(cache, x, x, [0, 7], [0]),                        # more rows than given
                 lambda: api.dlm_kv8_write(cache, x, x.float(), [0, 6], [0]),                # two types
                 lambda: api.dlm_kv8_write(cache, x, x.transpose(1, 2).contiguous().transpose(1, 2), [0, 6], [0]),
                 lambda: api.dlm_kv8_write(cache, x[:, :1], x[:, :1], [0, 6], [0]),
                 lambda: api.dlm_kv8_write(cache, x.half(), x.half(), [0, 6], [0]),
                 lambda: api.dlm_kv8_write(cache, x, x, [0], [0]),
                 lambda: api.dlm_kv8_read(cache, [0, 6], [0], k=x),
                 lambda: api.dlm_kv8_attention(cache, x[..., :32], [0, 6], [6]),
                 lambda: api.dlm_kv8_attention(cache, x, [0, 6], [6], out=torch.empty_like(x)[:5]),
                 lambda: api.dlm_kv8_attention(cache, x, [0, 6], [6], mask=torch.ones(6, 1, device=device)),
                 lambda: api.dlm_kv8_attention(cache, x, [0, 6], [6], mask=torch.ones(5, 1, dtype=torch.int32, device=device)),
                 lambda: api.dlm_qk_norm_rope(x.flatten(1), pos[:5], 1, 1, 64),
                 lambda: api.dlm_qk_norm_rope(x.flatten(1), pos.long(), 1, 1, 64),
                 lambda: api.dlm_qk_norm_rope(x.flatten(1), pos, 2, 1, 64),
                 lambda: api.dlm_qk_norm_rope(x.flatten(1), pos, 1, 1, 64, q_gain=torch.ones(64, device=device))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: api.dlm_kv8_write(cache, x, x, [0, 6], [60]),
                 lambda: api.dlm_kv8_write(cache, x, x, [0, 3, 6], [0, 9], [1, 1]),
                 lambda: api.dlm_kv8_read(cache, [0, 6], [0], [2]),
                 lambda: api.dlm_kv8_attention(cache, x, [0, 6], [65]),
                 lambda: api.dlm_kv8_attention(cache, x, [0, 6], [6], out=x),
                 lambda: api.dlm_kv8_attention(cache, x, [0, 6], [5], mask=torch.ones(6, 1, dtype=torch.int32, device=device)),
                 lambda: api.dlm_kv8_attention(long, x, [0, 6], [2000], workspace=torch.empty(16, dtype=torch.uint8, device=device)),
                 lambda: api.dlm_qk_norm_rope(x.flatten(1), pos, 1, 1, 64, eps=0.0)):
        with pytest.raises(api.DlmError):
            call()
    torch.cuda.synchronize()
    assert (api.dlm_kv8_read(cache, [0, 64], [0])[0] == 0).all()  # nothing was written by a refused call
