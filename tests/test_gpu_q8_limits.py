"""The 8-bit integer layers on the GPU at the edges of what they take, against the 64-bit oracle (oracle/q8.py).  Tolerances as in test_gpu_q8.py, whose helpers these
tests use (u = 2^-24, half a step of fp32)."""
import numpy as np
import pytest
import torch

from oracle import q8 as o_q8
from paper_2604_15750_amd import api
from test_gpu_q8 import BF16, F32, HALF_STEP, I8, U, VARIANTS, _coded, _columns, _gen, _np64, _untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [40, 4096, 40000])
def test_a_scale_whose_row_times_the_norm_is_past_fp32(device, dtype, width):
    """One value of a row far above the rest: max|t| rsqrt(mean(h^2) + eps) is up to sqrt(width) times the gain, 127 times what the scale is."""
    x = torch.randn(6, width, generator=_gen(width, 3)) * 1e-3
    x[:, 7] = torch.tensor([1.0, -1.0, 0.25, 3.0, -8.0, 100.0])
    for gain in (2.0 ** 90, 2.0 ** 99, 2.0 ** 101, 2.0 ** 120, 2.0 ** 123, 2.0 ** 127):
        xd, g = x.to(dtype), torch.full((width,), gain).to(dtype)
        t = _np64(xd) * gain
        with np.errstate(over="ignore"):
            bad = ~np.isfinite(t.astype(np.float32)).all(1)  # (a product of h and the gain past fp32 is none)
        q, s, _ = o_q8.add_norm(_np64(xd), _np64(g), None, 1e-5, None)
        codes, scale, _ = api.dlm_add_norm_q8(_columns(xd, device)[0], g.to(device))
        scale = _np64(scale)
        assert np.isnan(scale[bad]).all() and (s[~bad] < torch.finfo(F32).max).all()
        assert (np.abs(scale - s)[~bad] <= 72 * U * s[~bad]).all(), (gain, scale, s)
        assert (codes.cpu().numpy() == np.where(bad[:, None], 0, q)).all()


@pytest.mark.parametrize("rows", [1, 5, 300])
@pytest.mark.parametrize("width", [200, 4000])
def test_columns_beside_their_source(device, rows, width):
    """What is written lies in columns of the matrix that is read: codes beside their values, outputs beside their codes."""
    step = -(-(3 * width + 64) // 16) * 16  # bytes a row: values, codes, 32 bytes on each side
    wide = torch.full((rows, step // 2), 3.0, dtype=BF16, device=device)
    x = wide[:, 16:16 + width]
    x.copy_(torch.randn(rows, width, generator=_gen(rows, width)))
    kept = x.clone()
    codes, scale = wide.view(I8)[:, 32 + 2 * width:32 + 3 * width], torch.empty(rows, device=device)
    for norm in (False, True):
        codes.fill_(9)
        if norm:
            gain = torch.ones(width, dtype=BF16, device=device)
            want, want_scale, _ = api.dlm_add_norm_q8(kept, gain)
            api.dlm_add_norm_q8(x, gain, codes=codes, scale=scale)
        else:
            want, want_scale = api.dlm_q8_rows(kept)
            api.dlm_q8_rows(x, codes=codes, scale=scale)
        assert torch.equal(codes, want) and torch.equal(scale, want_scale) and torch.equal(x, kept)
    # a product of the codes, into the columns where the values were
    c, w = _coded(_gen(width, 5), width, width)
    weight = api.Q8Weight(_columns(c, device)[0], w.to(device))
    out = api.dlm_q8_gemm(weight, want, want_scale)
    api.dlm_q8_gemm(weight, codes, scale, out=x)
    assert torch.equal(x, out) and torch.equal(codes, want)
    assert (wide[:, :16] == 3).all() and (wide.view(I8)[:, 32 + 3 * width:] == torch.full((1,), 3.0, dtype=BF16).view(I8).repeat(step)[:step - 32 - 3 * width].to(device)).all()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,n,k", [v for v in VARIANTS if api.plan_q8_gemm(*v)["splits"] > 1])
def test_a_split_product_whatever_the_workspace_holds(device, rows, n, k, gated):
    """Each time against 64 bits, and bit for bit the same: sums of integers have no order."""
    n += gated and n % 2
    g = _gen(rows, n, k, 3)
    (q, s), (c, w) = _coded(g, rows, k, 0.3), _coded(g, n, k, 0.3)
    w = w * 30
    weight = api.Q8Weight(_columns(c, device)[0], w.to(device), gated=gated)
    qd, ws, first = _columns(q, device)[0], weight.workspace(rows), None
    # (the sums in 64 bits on the GPU: exact, as they are below 2^53)
    y = (q.to(device).double() @ c.to(device).double().t().contiguous()).cpu().numpy() * _np64(s)[:, None] * _np64(w)
    want, off = y, 3 * U * np.abs(y)
    if gated:
        want = o_q8.gated(y)
        off = (13 + 6 * np.abs(y[:, :n // 2])) * U * np.abs(want) + 2.0 ** -125 * np.abs(y[:, :n // 2] * y[:, n // 2:])
    for fill in (255, 127, 128, 0):
        out, wide = _columns(torch.full((rows, weight.outputs), 9.0), device)
        ws.fill_(fill)
        api.dlm_q8_gemm(weight, qd, s.to(device), out=out, workspace=ws)
        assert (np.abs(_np64(out) - want) <= off * (1 + 2.0 ** -7) + U * np.abs(want) + 2.0 ** -149).all() and _untouched(wide, weight.outputs)
        first = out if first is None else first
        assert torch.equal(out, first)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [4, 60, 700])
def test_the_gated_unit_where_it_is_large_and_small(device, dtype, rows):
    """Gates from -115 to 115 with up values from 2^-60 to 2^100: off by (13 + 6 |g|) u of the output and 2^-125 |g u| at most, besides the output's rounding.
    The latter is the whole of it below g = -87.3, where exp(-g) is past 2^126 and its reciprocal may be taken as zero."""
    f = 256
    g = _gen(rows, 71)
    codes = torch.zeros(2 * f, 16, dtype=I8)
    codes[:f, 0] = torch.randint(-115, 116, (f,), generator=g, dtype=torch.int16).to(I8)
    codes[:6, 0] = torch.tensor([-90, -89, -88, -87, 88, 115], dtype=I8)
    codes[f:, 1] = torch.randint(-127, 128, (f,), generator=g, dtype=torch.int16).to(I8)
    w = torch.ones(2 * f)
    w[f:] = torch.exp2(torch.randint(-60, 101, (f,), generator=g).float())
    w[f:f + 4] = 2.0 ** 100
    q = torch.zeros(rows, 16, dtype=I8)
    q[:, :2] = 1
    s = 1 - torch.rand(rows, generator=g) / 64  # (gates between the whole numbers)
    s[0] = 1
    out = api.dlm_q8_gemm(api.Q8Weight(codes.to(device), w.to(device), gated=True), q.to(device), s.to(device), dtype=dtype)
    y = o_q8.product(q.numpy(), _np64(s), codes.numpy(), _np64(w))
    want, size = o_q8.gated(y), np.abs(y[:, :f])
    off = ((13 + 6 * size) * U * np.abs(want) + 2.0 ** -125 * size * np.abs(y[:, f:])) * (1 + 2.0 ** -7)
    # the output's rounding: half a step, which below 2^-126 is 2^-150 in fp32 and, with 7 bits of fraction, 2^-134 in bf16
    off += HALF_STEP[dtype] * np.abs(want) + (2.0 ** -134 if dtype == BF16 else 2.0 ** -149)
    bad = ~(np.abs(_np64(out) - want) <= off)
    assert not bad.any(), (np.argwhere(bad)[:5], _np64(out)[bad][:5], want[bad][:5])
