"""The 8-bit integer linear layers on the GPU against the 64-bit oracle (oracle/q8.py).

Tolerances, derived before the first run (u = 2^-24, half a step of fp32; a rounding to bf16 is off by at most 2^-8 of the value):
  codes    none: the definition fixes them
  h        none: one addition in fp32, one rounding
  scale    of rows: one quotient, u (2 u are allowed).  Of a norm: a sum of squares over at most 128 additions in a row is off by 129 u of itself (its
           terms are positive), which the root halves; the division by the width, eps, the root (2 u) and two products: 72 u.  Below fp32's
           normal numbers, half of their step, 2^-150
  product  the sum is exact; its conversion and two products, 3 u; then the output's rounding
  gated    g and u are 3 u off.  d log(silu)/dg is at most 1 + |g| in size, so g's own error counts 3 (1 + |g|) u; the exponential's argument is rounded
           (|g| u, and its product with log2 e another |g| u), the exponential itself 2 u, the sum u, the reciprocal 2 u, two products 2 u, u's own 3 u:
           (13 + 6 |g|) u; below a reciprocal of 2^-126 it may be zero: 2^-125 |g u|; then the output's rounding
"""
import math

import numpy as np
import pytest
import torch

from oracle import q8 as o_q8
from paper_2604_15750_amd import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32, I8 = torch.bfloat16, torch.float32, torch.int8
HALF_STEP = {BF16: 2.0 ** -8, F32: U}


def _np64(t):
    return t.detach().cpu().double().numpy()


def _gen(*key):
    return torch.Generator(device="cpu").manual_seed(sum(k * 7919 ** i for i, k in enumerate(key)) % (1 << 62))


def _columns(x, device, gap=32, fill=3):
    """x on the device as columns of a wider matrix, at a stride of a multiple of 16 bytes: (the view, the whole)."""
    step = 16 // x.element_size()
    wide = torch.full((x.shape[0], -(-x.shape[1] // step) * step + 2 * gap), fill, dtype=x.dtype)
    wide[:, gap:gap + x.shape[1]] = x
    wide = wide.to(device)
    return wide[:, gap:gap + x.shape[1]], wide


def _untouched(wide, width, gap=32, fill=3):
    return bool((wide[:, :gap] == fill).all() and (wide[:, gap + width:] == fill).all())


def _rounded(dtype):
    """fp32 numpy -> the type -> fp64."""
    return lambda h: torch.from_numpy(np.ascontiguousarray(h)).to(dtype).double().numpy()


# ---- rows and norm -------------------------------------------------------------------------------------------------------------------

def _rows(g, rows, width, dtype):
    """Rows of different sizes, with values at the borders of their codes: halves of the maximum, and (k + 1/2) / 127 of it."""
    x = torch.randn(rows, width, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    for r in range(rows):
        top = float(x[r].abs().max())
        if r % 3 == 1:
            top = 127 * 2.0 ** math.floor(math.log2(top) - 4)
            k = torch.randint(-126, 126, (width,), generator=g) + 0.5
            x[r] = torch.where(torch.rand(width, generator=g) < 0.5, k * (top / 127), x[r].clamp(-top, top))
        if width > 3:
            x[r, r % width] = -top if r % 2 else top
            x[r, (r + 2) % width] = top / 2
    return x.to(dtype)


WIDTHS = [1, 7, 8, 64, 513, 1024, 2049, 4096, 5003, 8200, 16384, 16392, 32775, 70001]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [1, 5, 9])
def test_rows(device, dtype, width, rows):
    x = _rows(_gen(width, rows), rows, width, dtype)
    xd, _ = _columns(x, device)
    codes, wide = _columns(torch.full((rows, width), 9, dtype=I8), device)
    scale = torch.full((rows + 2,), 5.0, device=device)
    api.dlm_q8_rows(xd, codes=codes, scale=scale[1:rows + 1])
    q, s = o_q8.quantise(_np64(x))
    assert (codes.cpu().numpy() == q).all()
    assert (np.abs(_np64(scale)[1:-1] - s) <= 2 * U * s).all() and scale[0] == 5 and scale[-1] == 5
    assert _untouched(wide, width)
    again = api.dlm_q8_rows(xd)
    assert torch.equal(again[0], codes) and torch.equal(again[1], scale[1:rows + 1])


@pytest.mark.parametrize("dtype,h_dtype", [(BF16, None), (F32, None), (BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [1, 6])
def test_add_norm(device, dtype, h_dtype, width, rows):
    g = _gen(width, rows, 7)
    x, gain = _rows(g, rows, width, dtype), (1 + 0.3 * torch.randn(width, generator=g)).to(dtype)
    res = None if h_dtype is None else (2 * torch.randn(rows, width, generator=g)).to(h_dtype)
    xd, _ = _columns(x, device)
    eps = 1e-3
    q, s, h = o_q8.add_norm(_np64(x), _np64(gain), None if res is None else _np64(res), eps, _rounded(h_dtype))
    want = torch.from_numpy(h).to(h_dtype or dtype)

    def check(codes, scale, got):
        assert (codes.cpu().numpy() == q).all()
        assert (np.abs(_np64(scale) - s) <= 72 * U * s + 2.0 ** -150).all()
        assert torch.equal(got.cpu(), want)

    check(*api.dlm_add_norm_q8(xd, gain.to(device), None if res is None else res.to(device) if width % 8 == 0 else _columns(res, device)[0], eps=eps))
    if res is None:
        return
    # outputs given: columns of wider matrices; then in place, over the residual and over x
    hd, hw = _columns(torch.full((rows, width), 9.0, dtype=h_dtype), device)
    codes, cw = _columns(torch.full((rows, width), 9, dtype=I8), device)
    rd, rw = _columns(res, device)
    scale = torch.empty(rows, device=device)
    out = api.dlm_add_norm_q8(xd, gain.to(device), rd, h=hd, eps=eps, codes=codes, scale=scale)
    assert out[0] is codes and out[1] is scale and out[2] is hd
    check(*out)
    assert _untouched(hw, width) and _untouched(cw, width) and torch.equal(rd.cpu(), res)
    check(*api.dlm_add_norm_q8(xd, gain.to(device), rd, h=rd, eps=eps, codes=codes, scale=scale))
    assert _untouched(rw, width)
    if h_dtype == dtype:
        check(*api.dlm_add_norm_q8(xd, gain.to(device), _columns(res, device)[0], h=xd, eps=eps))


def test_the_smallest_the_largest_and_what_is_none(device):
    """Rows of zeros, of the least and greatest magnitudes, with NaN and infinities; a sum of squares past fp32; each leaves the others alone."""
    big = float(torch.finfo(F32).max)
    t = torch.zeros(10, 40)
    t[1, :3] = torch.tensor([1e-45, -3e-45, 2e-45])
    t[2] = torch.linspace(-1, 1, 40) * 2.0 ** -126
    t[3] = torch.linspace(-1, 1, 40) * big
    t[4, 5], t[5, 6], t[6, 7] = math.nan, math.inf, -math.inf
    t[7], t[8], t[9] = 2.0 ** -61 * torch.linspace(-1, 1, 40), 2.0 ** -59 * torch.linspace(1, -1, 40), torch.linspace(-3, 3, 40)
    q, s = o_q8.quantise(t.numpy())
    codes, scale = api.dlm_q8_rows(t.to(device))
    assert (codes.cpu().numpy() == q).all()
    assert np.array_equal(np.isnan(s), np.isnan(_np64(scale)))
    good = ~np.isnan(s)
    assert (np.abs(_np64(scale) - s)[good] <= 2 * U * s[good] + 2.0 ** -150).all()
    gain = torch.ones(40, device=device)
    codes, scale, _ = api.dlm_add_norm_q8(t.to(device), gain, eps=1e-5)
    bad = np.array([3, 4, 5, 6])  # (the squares of the third are past fp32's range)
    assert np.isnan(_np64(scale)[bad]).all() and (codes.cpu().numpy()[bad] == 0).all()
    rest = np.setdiff1d(np.arange(10), bad)
    q, s, _ = o_q8.add_norm(t.numpy()[rest], np.ones(40), None, 1e-5, None)
    assert (codes.cpu().numpy()[rest] == q).all() and (np.abs(_np64(scale)[rest] - s) <= 72 * U * s + 2.0 ** -150).all()
    # a gain that is NaN or infinite reaches every row; an infinite residual its own
    codes, scale, _ = api.dlm_add_norm_q8(t.to(device), gain * math.inf)
    assert torch.isnan(scale).all() and (codes == 0).all()
    res = torch.zeros(10, 40, device=device)
    res[9, 39] = math.inf
    _, scale, h = api.dlm_add_norm_q8(t.to(device), gain, res)
    assert list(torch.isnan(scale).cpu().numpy().nonzero()[0]) == [3, 4, 5, 6, 9] and torch.isinf(h[9, 39])


# ---- product -------------------------------------------------------------------------------------------------------------------------

def _coded(g, rows, width, spread=1.0):
    q = torch.randint(-127, 128, (rows, width), generator=g, dtype=torch.int16).to(I8)
    return q, torch.exp(spread * torch.randn(rows, generator=g)) / 127 / math.sqrt(width)


def _check_product(out, q, s, c, w, gated, dtype):
    y = o_q8.product(q.numpy(), _np64(s), c.numpy(), _np64(w))
    if gated:
        f = y.shape[1] // 2
        size = np.abs(y[:, :f])
        want = o_q8.gated(y)
        off = (13 + 6 * size) * U * np.abs(want) + 2.0 ** -125 * np.abs(y[:, :f] * y[:, f:])
    else:
        want, off = y, 3 * U * np.abs(y)
    off = off * (1 + 2.0 ** -7) + HALF_STEP[dtype] * np.abs(want) + 2.0 ** -149  # (second-order terms; the step of the smallest numbers)
    bad = ~(np.abs(_np64(out) - want) <= off)
    assert not bad.any(), (np.argwhere(bad)[:5], _np64(out)[bad][:5], want[bad][:5])


SHAPES = [(1, 1), (2, 16), (5, 3), (16, 64), (31, 17), (32, 63), (33, 65), (64, 256), (100, 777), (1003, 130), (260, 1000), (513, 2048), (96, 5000)]
ROWS = [1, 3, 16, 17, 33, 64, 65, 128, 200, 257]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("gated", [False, True])
def test_product(device, dtype, n, k, gated):
    if gated:
        n += n % 2
    g = _gen(n, k, gated)
    c, w = _coded(g, n, k)
    weight = api.Q8Weight(_columns(c, device)[0], (w * math.sqrt(k)).to(device), gated=gated)
    for rows in ROWS:
        q, s = _coded(g, rows, k)
        s = s * math.sqrt(k) * 0.1
        out, wide = _columns(torch.full((rows + 2, weight.outputs), 9.0, dtype=dtype), device)
        got = api.dlm_q8_gemm(weight, _columns(q, device)[0], s.to(device), out=out[:rows])
        print(rows, n, k, flush=True)
        _check_product(got, q, s, c, w * math.sqrt(k), gated, dtype)
        assert _untouched(wide, weight.outputs) and (out[rows:] == 9).all()


# rows that fill several tiles of every kind, and shapes of more than one round of workgroups
WIDE = [(300, 4096, 1024), (515, 1000, 4100), (1030, 2080, 520), (130, 12288, 300), (2300, 1500, 200), (8, 50000, 130)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n,k", WIDE)
@pytest.mark.parametrize("gated", [False, True])
def test_wide_product(device, dtype, rows, n, k, gated):
    g = _gen(rows, n, k)
    (q, s), (c, w) = _coded(g, rows, k, 0.3), _coded(g, n, k, 0.3)
    w = w * 30
    weight = api.Q8Weight(c.to(device) if k % 16 == 0 else _columns(c, device)[0], w.to(device), gated=gated)
    out, wide = _columns(torch.full((rows, weight.outputs), 9.0, dtype=dtype), device)
    ws = weight.workspace(rows + 100)
    for _ in range(2):  # (the second call finds what the first left in the workspace)
        out.fill_(9)
        api.dlm_q8_gemm(weight, _columns(q, device)[0], s.to(device), out=out, workspace=ws)
        # (the sums in 64 bits on the GPU: exact, as they are below 2^53)
        sums = (q.to(device).double() @ c.to(device).double().t().contiguous()).cpu().numpy()
        y = sums * _np64(s)[:, None] * _np64(w)
        want, off = y, 3 * U * np.abs(y)
        if gated:
            f = n // 2
            want = o_q8.gated(y)
            off = (13 + 6 * np.abs(y[:, :f])) * U * np.abs(want) + 2.0 ** -125 * np.abs(y[:, :f] * y[:, f:])
        off = off * (1 + 2.0 ** -7) + HALF_STEP[dtype] * np.abs(want) + 2.0 ** -149
        assert (np.abs(_np64(out) - want) <= off).all() and _untouched(wide, weight.outputs)


# shapes whose plain product is a launch of each streamed form, of each tile and of each band, with and without a K split, with one row block and with more
VARIANTS = [(193, 12352, 128), (98, 16443, 200), (1364, 641, 8200), (103, 7169, 8200), (770, 4786, 128), (129, 16713, 128), (290, 2181, 16400),
            (129, 8083, 8200), (290, 16436, 128), (129, 33001, 128), (1412, 1324, 16400), (131, 16407, 8200), (1158, 582, 640), (6, 24621, 2100),
            (518, 485, 8200), (34, 32, 128), (32, 4130, 1003), (33, 33, 4100), (14, 33, 8200), (2745, 129, 128), (14, 16506, 640), (321, 452, 8200),
            (2311, 581, 128), (33, 24603, 128), (805, 577, 8200), (34, 12292, 8200), (2733, 323, 128), (33, 16469, 128), (587, 409, 8200), (36, 2691, 16400),
            (2305, 782, 128), (65, 16407, 128), (778, 769, 8200), (65, 2694, 16400), (257, 10992, 128), (65, 32870, 128), (1667, 513, 8200), (1, 33, 128),
            (1, 4106, 128), (1, 8195, 128), (17, 33, 128), (17, 4101, 128), (97, 36888, 128), (1347, 974, 16400), (193, 33111, 200), (878, 3339, 16400),
            (513, 8297, 128), (706, 1352, 16400), (515, 24663, 128), (2321, 3339, 16400), (196, 36534, 200), (978, 2703, 16400)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,n,k", VARIANTS)
def test_every_variant(device, rows, n, k, gated):
    n += gated and n % 2
    g = _gen(rows, n, k)
    (q, s), (c, w) = _coded(g, rows, k, 0.3), _coded(g, n, k, 0.3)
    w = w * 30
    weight = api.Q8Weight(_columns(c, device)[0], w.to(device), gated=gated)
    qd = _columns(q, device)[0]
    # (the sums in 64 bits on the GPU: exact, as they are below 2^53)
    y = (q.to(device).double() @ c.to(device).double().t().contiguous()).cpu().numpy() * _np64(s)[:, None] * _np64(w)
    want, off = y, 3 * U * np.abs(y)
    if gated:
        want = o_q8.gated(y)
        off = (13 + 6 * np.abs(y[:, :n // 2])) * U * np.abs(want) + 2.0 ** -125 * np.abs(y[:, :n // 2] * y[:, n // 2:])
    for dtype in (F32, BF16):
        out, wide = _columns(torch.full((rows, weight.outputs), 9.0, dtype=dtype), device)
        ws = weight.workspace(rows)
        for fill in (255, 127, None):  # (whatever a workspace holds)
            out.fill_(9)
            if ws is not None and fill:
                ws.fill_(fill)
            api.dlm_q8_gemm(weight, qd, s.to(device), out=out, workspace=ws)
        assert (np.abs(_np64(out) - want) <= off * (1 + 2.0 ** -7) + HALF_STEP[dtype] * np.abs(want) + 2.0 ** -149).all() and _untouched(wide, weight.outputs)


def test_the_largest_sums(device):
    """Every product -128 x -128, and 127 x -128: the longest sums that 32 bits hold."""
    k = 131071
    q = torch.full((3, k), -128, dtype=I8)
    q[1] = 127
    c = torch.full((2, k), -128, dtype=I8)
    c[1] = 127
    for rows in (3, 150):
        qr = q.repeat(rows // 3, 1)
        weight = api.Q8Weight(_columns(c, device)[0], torch.ones(2, device=device))
        out = api.dlm_q8_gemm(weight, _columns(qr, device)[0], torch.ones(rows, device=device), dtype=F32)
        want = (qr.double() @ c.double().t()).float()
        assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("rows", [7, 70, 300])
@pytest.mark.parametrize("gated", [False, True])
def test_nan_stays_in_its_row_and_channel(device, rows, gated):
    g = _gen(rows, 11)
    (q, s), (c, w) = _coded(g, rows, 200), _coded(g, 90, 200)
    clean = api.dlm_q8_gemm(api.Q8Weight(_columns(c, device)[0], w.to(device), gated), _columns(q, device)[0], s.to(device))
    s[3], w[50] = math.nan, math.nan
    q[3] = 0
    out = api.dlm_q8_gemm(api.Q8Weight(_columns(c, device)[0], w.to(device), gated), _columns(q, device)[0], s.to(device))
    nan = torch.zeros_like(out, dtype=torch.bool)
    nan[3] = True
    nan[:, 5 if gated else 50] = True
    assert torch.equal(torch.isnan(out), nan) and torch.equal(out[~nan], clean[~nan])


@pytest.mark.parametrize("rows", [5, 100])
def test_bytes_behind_a_row_do_not_matter(device, rows):
    k = 100
    g = _gen(rows, 13)
    (q, s), (c, w) = _coded(g, rows, k), _coded(g, 40, k)
    outs = []
    for fill in (0, 127, -128):
        qd, cd = (torch.full((x.shape[0], 112), fill, dtype=I8, device=device) for x in (q, c))
        qd[:, :k], cd[:, :k] = q.to(device), c.to(device)
        outs.append(api.dlm_q8_gemm(api.Q8Weight(cd[:, :k], w.to(device)), qd[:, :k], s.to(device), dtype=F32))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("rows", [8, 90, 400])
@pytest.mark.parametrize("gated", [False, True])
def test_a_row_does_not_depend_on_the_others(device, rows, gated):
    """Sums of integers have no order: a row of a batch is that row alone, bit for bit."""
    g = _gen(rows, 17)
    (q, s), (c, w) = _coded(g, rows, 1500), _coded(g, 600, 1500)
    weight = api.Q8Weight(_columns(c, device)[0], w.to(device), gated=gated)
    qd = _columns(q, device)[0]
    out = api.dlm_q8_gemm(weight, qd, s.to(device), dtype=F32)
    for r in (0, rows // 2, rows - 1):
        assert torch.equal(api.dlm_q8_gemm(weight, qd[r:r + 1], s[r:r + 1].to(device), dtype=F32)[0], out[r])


# ---- together, as a layer runs them --------------------------------------------------------------------------------------------------

def _layer(device, rows, d, f, seed):
    g = _gen(rows, d, f, seed)
    x, res = (torch.randn(rows, d, generator=g)).to(BF16).to(device), (3 * torch.randn(rows, d, generator=g)).to(device)
    gain = (1 + 0.2 * torch.randn(d, generator=g)).to(BF16).to(device)
    up = (0.05 * torch.randn(2 * f, d, generator=g)).to(device)
    down = (0.05 * torch.randn(d, f, generator=g)).to(BF16).to(device)
    return x, res, gain, up, down


class Layer:
    """A feed-forward layer with the memory that it keeps."""

    def __init__(self, device, rows, d, f, seed=0):
        self.x, self.res, self.gain, self.w_up, self.w_down = _layer(device, rows, d, f, seed)
        self.up, self.down = api.Q8Weight.quantise(self.w_up, gated=True), api.Q8Weight.quantise(self.w_down)
        self.ws = self.up.workspace(rows), self.down.workspace(rows)
        e = lambda *a, **k: torch.empty(*a, device=device, **k)  # noqa: E731
        self.h, self.act, self.out = e(rows, d), e(rows, f, dtype=BF16), e(rows, d, dtype=BF16)
        self.codes = e(rows, d, dtype=I8), e(rows, f, dtype=I8)
        self.scale = e(rows), e(rows)

    def run(self):
        api.dlm_add_norm_q8(self.x, self.gain, self.res, h=self.h, codes=self.codes[0], scale=self.scale[0])
        api.dlm_q8_gemm(self.up, self.codes[0], self.scale[0], out=self.act, workspace=self.ws[0])
        api.dlm_q8_rows(self.act, codes=self.codes[1], scale=self.scale[1])
        return api.dlm_q8_gemm(self.down, self.codes[1], self.scale[1], out=self.out, workspace=self.ws[1])


@pytest.mark.parametrize("rows", [1, 8, 70, 300])
@pytest.mark.parametrize("d,f", [(128, 384), (512, 1536)])
def test_a_layer(device, rows, d, f):
    """Each operator on what the ones before it left; and the layer as a whole against the same layer in 64 bits, unquantised: a code is off by half a
    step of a 127th of the row's maximum, so the two agree to about 1 % and are tied to each other loosely, far from an error's size."""
    L = Layer(device, rows, d, f)
    L.run()
    q, s, h = o_q8.add_norm(_np64(L.x), _np64(L.gain), _np64(L.res), 1e-5, _rounded(F32))
    assert (L.codes[0].cpu().numpy() == q).all() and (_np64(L.h) == h).all()
    cu, su = (t.cpu() for t in api.dlm_q8_rows(L.w_up))
    _check_product(L.act, L.codes[0].cpu(), L.scale[0], cu, su, True, BF16)
    q, s = o_q8.quantise(_np64(L.act))
    assert (L.codes[1].cpu().numpy() == q).all()
    cd, sd = (t.cpu() for t in api.dlm_q8_rows(L.w_down))
    _check_product(L.out, L.codes[1].cpu(), L.scale[1], cd, sd, False, BF16)
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + 1e-5) * _np64(L.gain)
    want = o_q8.gated(y @ _np64(L.w_up).T) @ _np64(L.w_down).T
    assert np.linalg.norm(_np64(L.out) - want) <= 0.05 * np.linalg.norm(want)


@pytest.mark.parametrize("rows", [8, 300])
def test_a_captured_layer_replays(device, rows):
    """Captured once, replayed on new inputs, with eager work of the same workspaces between the replays."""
    L = Layer(device, rows, 512, 1536)
    L.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.run()
    for i in range(4):
        x, res, _, _, _ = _layer(device, rows, 512, 1536, 10 + i)
        L.x.copy_(x)
        L.res.copy_(res)
        L.out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = L.out.clone(), L.h.clone()
        L.out.fill_(7)
        L.run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], L.out) and torch.equal(got[1], L.h)


def test_captured_products_share_a_workspace_or_have_none_given(device):
    """Two graphs whose products split K, replayed in turn on one workspace; and a third that makes a workspace of its own each time."""
    rows, n, k = 64, 512, 8192
    assert api.plan_q8_gemm(rows, n, k)["splits"] > 1
    made = []
    for i in range(2):
        g = _gen(i, 23)
        (q, s), (c, w) = _coded(g, rows, k), _coded(g, n, k)
        made.append((api.Q8Weight(c.to(device), w.to(device)), q.to(device), s.to(device)))
    ws = made[0][0].workspace(rows)
    want = [api.dlm_q8_gemm(*m, dtype=F32) for m in made]
    outs = [torch.empty_like(y) for y in want + want[:1]]
    graphs = []
    torch.cuda.synchronize()
    for i, m in enumerate(made + made[:1]):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            api.dlm_q8_gemm(*m, out=outs[i], workspace=ws if i < 2 else None)
    for _ in range(4):
        for y in outs:
            y.fill_(7)
        for graph in graphs:
            graph.replay()
        api.dlm_q8_gemm(*made[0], workspace=ws)
        torch.cuda.synchronize()
        for y, z in zip(outs, want + want[:1]):
            assert torch.equal(y, z)


def test_rows_far_apart(device):
    """A stride whose tiles would be past 32 bits."""
    rows, k, stride = 150, 100, (1 << 22) + 16
    g = _gen(29)
    (q, s), (c, w) = _coded(g, rows, k), _coded(g, 70, k)
    far = torch.zeros(rows * stride, dtype=I8, device=device).as_strided((rows, k), (stride, 1))
    far.copy_(q)
    weight = api.Q8Weight(_columns(c, device)[0], w.to(device))
    assert torch.equal(api.dlm_q8_gemm(weight, far, s.to(device), dtype=F32), api.dlm_q8_gemm(weight, _columns(q, device)[0], s.to(device), dtype=F32))


@pytest.mark.parametrize("rows,n", [(257, 300), (300, 24600), (40, 200)])
def test_rows_as_far_apart_as_a_tile_takes_them(device, rows, n):
    k, stride = 130, 1 << 22
    g = _gen(31, rows)
    (q, s), (c, w) = _coded(g, rows, k), _coded(g, n, k)
    far = torch.zeros(rows * stride, dtype=I8, device=device).as_strided((rows, k), (stride, 1))
    far.copy_(q)
    weight = api.Q8Weight(_columns(c, device)[0], w.to(device))
    assert torch.equal(api.dlm_q8_gemm(weight, far, s.to(device), dtype=F32), api.dlm_q8_gemm(weight, _columns(q, device)[0], s.to(device), dtype=F32))


def test_offsets_past_32_bits(device):
    """Rows 2^24 elements apart, 300 of them, as inputs and as outputs of every operator."""
    rows, width, stride = 300, 40, 1 << 24
    g = _gen(37)
    far = torch.zeros(rows * stride, dtype=BF16, device=device).as_strided((rows, width), (stride, 1))
    bytes_ = torch.zeros(rows * stride, dtype=I8, device=device).as_strided((rows, width), (stride, 1))
    x, res, gain = (torch.randn(rows, width, generator=g).to(BF16).to(device) for _ in range(3))
    far.copy_(x)
    scale = torch.empty(rows, device=device)
    want = api.dlm_q8_rows(x)
    api.dlm_q8_rows(far, codes=bytes_, scale=scale)
    assert torch.equal(bytes_, want[0]) and torch.equal(scale, want[1])
    want = api.dlm_add_norm_q8(x, gain[0], res)
    api.dlm_add_norm_q8(x, gain[0], res, h=far, codes=bytes_, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip((bytes_, scale, far), want))
    (c, w) = _coded(g, width, 64)
    weight = api.Q8Weight(c.to(device), w.to(device))
    q, s = (t.to(device) for t in _coded(g, rows, 64))
    api.dlm_q8_gemm(weight, q, s, out=far)
    assert torch.equal(far, api.dlm_q8_gemm(weight, q, s))


@pytest.mark.parametrize("rows", [3, 40, 150])
def test_the_most_channels(device, rows):
    """2^24 channels: a packed weight of 2 GiB, outputs past 2^31.  Sums of 16 products are exact in fp32, and the scales are powers of two."""
    n, k = 1 << 24, 16
    q = torch.randint(-128, 128, (rows, k), dtype=I8, generator=_gen(41, rows)).to(device)
    c = torch.randint(-128, 128, (n, k), dtype=I8, device=device, generator=torch.Generator(device=device).manual_seed(3))
    w = torch.exp2((torch.arange(n, device=device) % 7).float())
    weight = api.Q8Weight(c, w)
    out = api.dlm_q8_gemm(weight, q, torch.full((rows,), 0.5, device=device), dtype=F32)
    for lo in range(0, n, 1 << 20):  # (torch's product of 150 x 16 x 2^22 in fp32, 2.5 GB of output, is wrong in its rows behind 2 GiB: element by element the sums are ours)
        part = slice(lo, lo + (1 << 20))
        assert torch.equal(out[:, part], (q.float() @ c[part].float().t().contiguous()) * 0.5 * w[part])


@pytest.mark.parametrize("n,k", [(1, 1), (40, 16), (200, 130)])
def test_the_most_rows(device, n, k):
    rows = 1 << 20
    q = torch.zeros(rows, -(-k // 16) * 16, dtype=I8, device=device)
    q.random_(-128, 128, generator=torch.Generator(device=device).manual_seed(5))
    c, _ = _coded(_gen(43, n), n, k)
    weight = api.Q8Weight(_columns(c, device)[0], torch.ones(n, device=device))
    out = api.dlm_q8_gemm(weight, q[:, :k], torch.ones(rows, device=device), dtype=F32)
    assert torch.equal(out, q[:, :k].float() @ c.to(device).float().t().contiguous())
    with pytest.raises(api.DlmError, match="too many rows"):
        api.dlm_q8_gemm(weight, torch.zeros(rows + 1, q.shape[1], dtype=I8, device=device)[:, :k], torch.ones(rows + 1, device=device))


def test_two_streams_with_a_workspace_each(device):
    layers = [Layer(device, 64, 512, 4096, seed) for seed in (1, 2)]
    assert layers[0].ws[1] is not None
    want = [L.run().clone() for L in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for L, st in zip(layers, streams):
            with torch.cuda.stream(st):
                L.run()
    torch.cuda.synchronize()
    for L, w in zip(layers, want):
        assert torch.equal(L.out, w)
