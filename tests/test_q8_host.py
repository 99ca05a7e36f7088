"""Host-only checks of the 8-bit integer layers' entry points: sizes and refusals (no call gets as far as the GPU)."""
import ctypes as C

import pytest
import torch

from paper_2604_15750_amd import api

EINVAL, ESHAPE, ECAPACITY = -1, -2, -3
P = 1 << 40  # a pointer that is never dereferenced: validation fails first
Q, R, S, T = (P + (i << 36) for i in range(1, 5))  # others, far from it


def _err():
    return api.lib().dlm_last_error().decode()


def _weight(n=64, k=256, gated=0, data=T):
    return C.byref(api.dlm_q8_weight(n, k, gated, data))


def test_weight_bytes():
    f = api.lib().dlm_q8_weight_bytes
    assert C.sizeof(api.dlm_q8_weight) == 24
    # units of 32 channels x 128 k, and 32 scales each
    assert f(1, 1, 0) == 4096 + 128 and f(33, 129, 0) == 2 * (2 * 4096 + 128) and f(64, 64, 1) == 2 * (4096 + 128) and f(66, 128, 1) == 3 * (4096 + 128)
    assert f(1 << 17, 131071, 0) == 4096 * (1024 * 4096 + 128)  # (beyond 32 bits)
    for bad in ((0, 1, 0), (1, 0, 0), (3, 8, 1), (-2, 8, 1), (1, 131072, 0), ((1 << 24) + 1, 8, 0), (1 << 24, 131071, 0)):
        assert f(*bad) == 0, bad


def test_workspace_grows_with_rows():
    f = api.lib().dlm_q8_gemm_workspace
    for n, k, gated in ((4096, 12288, 0), (64, 131071, 0), (1000, 1000, 1), (24576, 4096, 1)):
        sizes = [f(r, n, k, gated) for r in (1, 2, 16, 17, 64, 65, 128, 300, 512, 1000, 5000, 1 << 20)]
        assert sizes == sorted(sizes) and all(s % 16 == 0 for s in sizes) and sizes[-1] < 1 << 31
    assert f(0, 64, 64, 0) == 0 and f(5, 0, 64, 0) == 0 and f(5, 3, 64, 1) == 0


def test_rows_refusals():
    f = api.lib().dlm_q8_rows

    def call(x=P, stride=256, rows=4, width=200, dtype=1, codes=Q, cs=208, scale=R):
        return f(x, stride, rows, width, dtype, codes, cs, scale, None)

    assert call(x=None) == call(codes=None) == call(scale=None) == EINVAL and "null" in _err()
    assert call(dtype=2) == EINVAL
    assert call(x=P + 2) == call(codes=Q + 8) == call(scale=R + 2) == EINVAL and "aligned" in _err()
    assert call(stride=199) == call(stride=204) == call(stride=-256) == call(cs=200) == call(cs=192) == EINVAL and "stride" in _err()
    assert call(rows=-1) == call(width=0) == call(width=(1 << 20) + 1, stride=1 << 21, cs=1 << 21) == ESHAPE
    assert call(rows=1 << 22) == ECAPACITY
    # x spans 3 * 512 + 400 bytes
    assert call(codes=P + 1920) == EINVAL and call(codes=P + 16) == EINVAL and call(scale=P + 1932) == EINVAL and call(scale=Q + 208) == EINVAL and "overlap" in _err()
    assert call(rows=0) == 0


def test_add_norm_refusals():
    f = api.lib().dlm_add_norm_q8

    def call(x=P, stride=256, rows=4, width=200, dtype=1, res=Q, rs=256, h=R, hs=256, hd=0, gain=S, eps=1e-5, codes=T, cs=208, scale=T + 4096):
        return f(x, stride, rows, width, dtype, res, rs, h, hs, hd, gain, eps, codes, cs, scale, None)

    assert call(x=None) == call(gain=None) == call(codes=None) == call(scale=None) == EINVAL
    assert call(res=None) == call(h=None) == EINVAL and "together" in _err()
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert call(eps=eps) == EINVAL and "eps" in _err()
    assert call(hd=2) == EINVAL and call(dtype=0, stride=256, hd=1) == EINVAL and call(dtype=2) == EINVAL
    assert call(gain=S + 2) == call(res=Q + 4) == call(h=R + 8) == EINVAL and "aligned" in _err()
    assert call(rs=199) == call(hs=202) == call(stride=252) == call(cs=199) == EINVAL
    assert call(width=0) == ESHAPE and call(rows=1 << 22) == ECAPACITY
    # what is written overlaps
    assert call(h=Q + 1024) == call(h=Q, hs=260) == EINVAL and "residual" in _err()
    assert call(h=P, hs=256, hd=0) == EINVAL and "overlaps x" in _err()  # (another type than x's)
    assert call(h=S) == call(gain=R + 16) == call(codes=S) == call(scale=S + 396) == call(codes=Q) == call(codes=R + 800) == call(scale=R) == call(scale=Q + 4) == EINVAL
    assert call(rows=0) == 0 and call(rows=0, res=None, h=None) == 0 and call(rows=0, h=Q) == 0 and call(rows=0, h=P, hd=1) == 0


def test_columns_of_one_matrix_do_not_overlap():
    f = api.lib().dlm_q8_rows  # 200 bf16 (400 bytes) and 200 codes side by side in rows of 640 bytes; zero rows: nothing is launched
    assert f(P, 320, 0, 200, 1, P + 400, 640, R, None) == 0
    g = api.lib().dlm_add_norm_q8
    args = lambda rows, h: (P, 512, rows, 200, 1, Q, 512, h, 512, 1, S, 1e-5, T, 208, T + (1 << 30), None)  # noqa: E731
    assert g(*args(4, Q + 384)) == EINVAL and g(*args(4, Q + 1024 - 384)) == EINVAL


def test_pack_refusals():
    f = api.lib().dlm_q8_weight_pack
    assert f(None, P, 256, R, None) == f(_weight(data=None), P, 256, R, None) == f(_weight(), None, 256, R, None) == f(_weight(), P, 256, None, None) == EINVAL
    assert f(_weight(data=T + 8), P, 256, R, None) == f(_weight(), P + 8, 256, R, None) == f(_weight(), P, 256, R + 1, None) == EINVAL
    assert f(_weight(gated=2), P, 256, R, None) == EINVAL and f(_weight(), P, 255, R, None) == f(_weight(), P, 264, R, None) == EINVAL
    assert f(_weight(n=63, gated=1), P, 256, R, None) == f(_weight(n=0), P, 256, R, None) == f(_weight(k=131072), P, 1 << 20, R, None) == ESHAPE
    assert f(_weight(), T + 1024, 256, R, None) == f(_weight(), P, 256, T + 64 * 256 + 128, None) == EINVAL and "overlap" in _err()


def test_gemm_refusals():
    f = api.lib().dlm_q8_gemm

    def call(w=None, x=P, stride=256, scale=Q, rows=4, out=R, os=64, dtype=1, ws=None, size=0):
        return f(w or _weight(), x, stride, scale, rows, out, os, dtype, ws, size, None)

    assert f(None, P, 256, Q, 4, R, 64, 1, None, 0, None) == EINVAL and call(_weight(data=None)) == EINVAL
    assert call(x=None) == call(scale=None) == call(out=None) == EINVAL and call(dtype=2) == EINVAL
    assert call(x=P + 8) == call(scale=Q + 2) == call(out=R + 4) == call(ws=S + 8, size=64) == EINVAL and "aligned" in _err()
    assert call(stride=255) == call(stride=264) == call(os=63) == call(os=68) == EINVAL and call(os=66, dtype=0) == EINVAL
    assert call(_weight(gated=2)) == EINVAL and call(_weight(n=65, gated=1)) == ESHAPE and call(rows=-1) == ESHAPE and call(rows=(1 << 20) + 1) == ECAPACITY
    assert call(out=P) == call(out=P + 1008) == call(scale=R) == call(scale=R + 508) == call(out=T) == EINVAL and "overlap" in _err()
    assert call(rows=0) == 0 and call(_weight(gated=1), os=32, rows=0) == 0
    n, k = 4096, 12288
    for rows in (1, 100, 486):
        need = api.plan_q8_gemm(rows, n, k)["workspace_kib"] << 10
        assert need <= api.lib().dlm_q8_gemm_workspace(rows, n, k, 0)
        if need:
            big = _weight(n, k)
            args = dict(w=big, stride=k, os=n, rows=rows)
            assert call(**args) == call(ws=S, size=need - 16, **args) == ECAPACITY and "workspace" in _err()
            assert call(ws=P, size=need, **args) == call(ws=R, size=need, **args) == call(ws=T, size=need, **args) == EINVAL and "workspace" in _err()


def test_plans():
    """What is asked for is what is launched; a workspace for more rows serves fewer."""
    f = api.lib().dlm_plan_q8_gemm
    out = (C.c_int32 * 6)()
    assert f(8, 64, 64, 0, None) == EINVAL and f(8, 64, 64, 2, out) == EINVAL
    for bad in ((0, 64, 64), (8, 0, 64), (8, 64, 131072), ((1 << 20) + 1, 64, 64)):
        assert f(*bad, 0, out) == ESHAPE
    for n, k, gated in ((4096, 12288, False), (640, 131071, False), (1000, 3000, True), (12288, 4096, False), (33, 65, False), (8232, 16400, False), (30000, 131071, False)):
        for rows in (1, 16, 17, 32, 33, 64, 96, 130, 194, 300, 700, 2000, 20000):
            p = api.plan_q8_gemm(rows, n, k, gated)
            assert (p["kernel"] != "streamed" or rows <= 32) and p["splits"] >= 1 and p["workgroups"] >= p["splits"]
            assert (p["workspace_kib"] > 0) == (p["splits"] > 1)
            for more in (rows, rows + 1, rows + 500):
                assert p["workspace_kib"] << 10 <= api.lib().dlm_q8_gemm_workspace(more, n, k, int(gated))


def test_every_variant_is_reached_by_a_test():
    from test_gpu_q8 import VARIANTS

    plans = [(v[0], api.plan_q8_gemm(*v)) for v in VARIANTS]
    tiles = {(128, 256), (128, 384), (192, 128), (192, 384), (256, 256)}
    bands = {(32, 64), (32, 96), (32, 128), (64, 96), (64, 128), (96, 128), (96, 192), (128, 128), (160, 128), (160, 192)}
    assert {(p["kernel"], p["rows"], p["cols"]) for _, p in plans if p["splits"] == 1} == {("tiled", *t) for t in tiles} | {("banded", *b) for b in bands} | \
        {("streamed", 16, c) for c in (16, 32, 48)} | {("streamed", 32, c) for c in (16, 32)}
    assert {(p["kernel"], p["rows"], p["cols"]) for _, p in plans if p["splits"] > 1} == {("tiled", *t) for t in tiles} | {("banded", *b) for b in bands}
    # a band's W is read in another way where one row block reads it
    for one in (False, True):
        assert {(p["rows"], p["cols"]) for m, p in plans if p["kernel"] == "banded" and (m <= p["rows"]) == one} == bands


def test_python_refusals(monkeypatch):
    """Shapes, types and memory that the library could not see."""
    monkeypatch.setattr(api, "_device", lambda: -1)  # (tensors here are on the CPU, whose index is -1)
    monkeypatch.setattr(api, "_gpu_of", lambda name, t: -1)
    monkeypatch.setattr(api, "_stream", lambda: 0)
    x, gain = torch.zeros(4, 64), torch.ones(64)
    for bad in (dict(codes=torch.zeros(4, 64)), dict(codes=torch.zeros(3, 64, dtype=torch.int8)), dict(codes=torch.zeros(4, 80, dtype=torch.int8)),
                dict(scale=torch.zeros(4, dtype=torch.float64)), dict(scale=torch.zeros(5)), dict(scale=torch.zeros(8)[::2])):
        with pytest.raises(ValueError):
            api.dlm_q8_rows(x, **bad)
        with pytest.raises(ValueError):
            api.dlm_add_norm_q8(x, gain, **bad)
    with pytest.raises(ValueError):
        api.dlm_q8_rows(x.half())
    with pytest.raises(ValueError):
        api.dlm_q8_rows(x[:, ::2])
    with pytest.raises(ValueError):
        api.dlm_q8_rows(x[0])
    for bad in (dict(residual=torch.zeros(4, 64).bfloat16()), dict(residual=torch.zeros(3, 64)), dict(h=torch.zeros(4, 64)),
                dict(residual=torch.zeros(4, 64), h=torch.zeros(4, 64).bfloat16()), dict(residual=torch.zeros(4, 64), h=torch.zeros(4, 65))):
        with pytest.raises(ValueError):
            api.dlm_add_norm_q8(x, gain, **bad)
    with pytest.raises(ValueError):
        api.dlm_add_norm_q8(x, gain.bfloat16())
    codes = torch.zeros(4, 64, dtype=torch.int8)
    with pytest.raises(ValueError):
        api.Q8Weight(codes, torch.zeros(5))
    with pytest.raises(ValueError):
        api.Q8Weight(codes.int(), torch.zeros(4))
    with pytest.raises(api.DlmError, match="ESHAPE"):
        api.Q8Weight(codes[:3], torch.zeros(3), gated=True)
    # the last row's bytes up to a multiple of 16 are behind the tensor's memory
    with pytest.raises(ValueError, match="multiple of 16"):
        api.Q8Weight(torch.zeros(4 * 48 - 1, dtype=torch.int8).as_strided((4, 40), (48, 1)).as_strided((4, 40), (48, 1), 7), torch.zeros(4))

    class W:
        n, k, outputs, gated, _data, _ref = 32, 64, 32, False, torch.zeros(1), 0
        workspace = staticmethod(lambda rows: None)

    s = torch.zeros(4)
    for bad in (dict(x=codes[:, :48]), dict(x=codes.int()), dict(x_scale=torch.zeros(3)), dict(out=torch.zeros(4, 33)), dict(out=torch.zeros(5, 32)),
                dict(out=torch.zeros(4, 32).half()), dict(workspace=torch.zeros(64)[::2])):
        with pytest.raises(ValueError):
            api.dlm_q8_gemm(W, **{**dict(x=codes, x_scale=s), **bad})


def test_calls_without_rows_return(monkeypatch):
    monkeypatch.setattr(api, "_device", lambda: -1)
    monkeypatch.setattr(api, "_gpu_of", lambda name, t: -1)
    monkeypatch.setattr(api, "_stream", lambda: 0)
    codes, scale = api.dlm_q8_rows(torch.zeros(0, 64))
    assert codes.shape == (0, 64) and scale.shape == (0,)
    assert api.dlm_add_norm_q8(torch.zeros(0, 64), torch.ones(64), torch.zeros(0, 64))[2].shape == (0, 64)
