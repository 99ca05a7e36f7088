"""The 8-bit integer layers on the GPU at the edges of what they take, against the 64-bit oracle (oracle/q8.py).  Tolerances as in test_gpu_q8.py, whose helpers these
tests use (u = 2^-24, half a step of fp32)."""
import numpy as np
import pytest
import torch

from oracle import q8 as o_q8
from paper_2604_15750_amd import api
from test_gpu_q8 import BF16, F32, U, _columns, _gen, _np64

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
