"""The Python calls of the 8-bit integer layers: the extension and the way through ctypes make the same C call, or refuse alike; and the extension is optional."""
import ctypes as C
import sys

import pytest
import torch

from paper_2604_15750_amd import api, build

VP, I32, I64, F32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
ROWS = C.CFUNCTYPE(I32, VP, I64, I32, I32, I32, VP, I64, VP, VP)
NORM = C.CFUNCTYPE(I32, VP, I64, I32, I32, I32, VP, I64, VP, I64, I32, VP, F32, VP, I64, VP, VP)
GEMM = C.CFUNCTYPE(I32, VP, VP, I64, VP, I32, VP, I64, I32, VP, C.c_size_t, VP)
BF, I8 = torch.bfloat16, torch.int8


@pytest.fixture
def both(monkeypatch):
    """both(f): what f's call hands to the library through the extension and through ctypes, or the exceptions' types; both.taken: whether
    the extension made the call itself.  CPU tensors stand for the GPU's (index -1); nothing is launched."""
    ext = api._q8_calls()
    assert ext is not None, "the extension has not been built"
    L, seen = api.lib(), []

    class Both:
        status = 0

        def __call__(self, f):
            out = []
            for through in (True, False):
                seen.clear()
                self.taken = False
                monkeypatch.setattr(api, "_q8_calls", (lambda: Spy) if through else (lambda: None))
                try:
                    f()
                    out.append(list(seen))
                except Exception as e:  # noqa: BLE001
                    out.append(type(e))
                if through:
                    taken = self.taken
            self.taken = taken
            return out

    self = Both()

    def call(*a):
        seen.append(a)
        return self.status

    calls = [t(call) for t in (ROWS, NORM, GEMM)]

    class Recorder:
        dlm_q8_rows, dlm_add_norm_q8, dlm_q8_gemm = calls
        dlm_q8_gemm_workspace, dlm_last_error = staticmethod(lambda *a: 0), L.dlm_last_error

    class Spy:
        @staticmethod
        def ask(f, args):
            rc = f(*args)
            self.taken = rc is not None
            assert self.taken == (len(seen) == 1)
            return rc

        rows, norm, gemm = (staticmethod(lambda *a, f=f: Spy.ask(f, a)) for f in (ext.rows, ext.norm, ext.gemm))

    real = [C.cast(f, VP).value for f in (L.dlm_q8_rows, L.dlm_add_norm_q8, L.dlm_q8_gemm)]
    for name, value in (("lib", lambda: Recorder), ("_device", lambda: -1), ("_stream", lambda: 0x1230), ("_gpu_of", lambda name, t: -1)):
        monkeypatch.setattr(api, name, value)
    ext.bind(*(C.cast(f, VP).value for f in calls))
    yield self
    ext.bind(*real)


def _z(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def test_rows_either_way(both):
    base = dict(x=_z(6, 48), codes=_z(6, 48, dtype=I8), scale=_z(6))
    for change, ok in (({}, True), (dict(x=_z(6, 48, dtype=BF)), True), (dict(x=_z(6, 80)[:, 4:52], codes=_z(6, 96, dtype=I8)[:, 16:64]), True), (dict(x=_z(6, 48).half()), False),
                       (dict(x=_z(48, 6).t()), False), (dict(x=_z(5, 48)), False), (dict(x=_z(6, 47)), False), (dict(x=_z(48)), False), (dict(codes=_z(6, 48)), False),
                       (dict(codes=_z(6, 49, dtype=I8)), False), (dict(scale=_z(5)), False), (dict(scale=_z(12)[::2]), False), (dict(scale=_z(6, dtype=BF)), False),
                       (dict(scale=_z(6, 1)), False)):
        a, b = both(lambda: api.dlm_q8_rows(**dict(base, **change)))
        assert a == b and both.taken == ok and (type(a) is list) == ok, change
    for x in (_z(1, 45), _z(2, 80)[:1, :45], _z(1, 45, dtype=BF)):  # a single row's stride holds it in multiples of 16 bytes
        a, b = both(lambda: api.dlm_q8_rows(x, _z(1, 45, dtype=I8), base["scale"][:1]))
        assert [c[1:5] + c[6:7] for c in a] == [c[1:5] + c[6:7] for c in b] == [(48, 1, 45, 0 if x.dtype != BF else 1, 48)] and both.taken
    assert [c[2:5] for c in both(lambda: api.dlm_q8_rows(base["x"]))[1]] == [(6, 48, 0)] and not both.taken  # (new outputs: not the extension's)
    both.status = -2
    assert both(lambda: api.dlm_q8_rows(**base)) == [api.DlmError, api.DlmError] and both.taken


def test_add_norm_either_way(both):
    base = dict(x=_z(6, 48, dtype=BF), gain=_z(48, dtype=BF), residual=_z(6, 48), h=_z(6, 48), eps=1e-5, codes=_z(6, 48, dtype=I8), scale=_z(6))
    res = base["residual"]
    for change, ok in (({}, True), (dict(residual=None, h=None), True), (dict(h=res), True), (dict(residual=_z(6, 48, dtype=BF), h=base["x"]), True),
                       (dict(residual=_z(6, 80)[:, 4:52], h=_z(6, 64)[:, :48]), True), (dict(h=_z(6, 48, dtype=BF)), False), (dict(residual=_z(5, 48)), False),
                       (dict(residual=_z(6, 48).half(), h=_z(6, 48).half()), False), (dict(x=_z(6, 48), gain=_z(48), residual=_z(6, 48, dtype=BF), h=_z(6, 48, dtype=BF)), False),
                       (dict(residual=None), False), (dict(gain=_z(48)), False), (dict(gain=_z(47, dtype=BF)), False), (dict(gain=_z(96, dtype=BF)[::2]), False),
                       (dict(h=_z(6, 47)), False), (dict(codes=_z(7, 48, dtype=I8)), False), (dict(scale=_z(7)), False)):
        a, b = both(lambda: api.dlm_add_norm_q8(**dict(base, **change)))
        assert a == b and both.taken == ok and (type(a) is list) == ok, change
    a, b = both(lambda: api.dlm_add_norm_q8(**dict(base, eps=1)))
    assert a == b and len(a) == 1 and not both.taken
    assert len(both(lambda: api.dlm_add_norm_q8(**dict(base, h=None)))[1]) == 1 and not both.taken  # (a new h)


@pytest.mark.parametrize("k", [64, 40])
@pytest.mark.parametrize("gated", [False, True])
def test_gemm_either_way(both, k, gated):
    n = 24
    data = _z(64, dtype=torch.uint8)
    desc = api.dlm_q8_weight(n, k, int(gated), data.data_ptr())

    class W:
        outputs, _data, _ref = n // 2 if gated else n, data, C.addressof(desc)
        workspace = staticmethod(lambda rows: None)

    W.k = k
    x = _z(6, 64, dtype=I8)[:, :k]
    base = dict(weight=W, x=x, x_scale=_z(6), out=_z(6, W.outputs))
    for change, ok in (({}, True), (dict(out=_z(6, 64, dtype=BF)[:, 8:8 + W.outputs]), True), (dict(workspace=_z(64, dtype=torch.uint8)), True), (dict(workspace=_z(16)), True),
                       (dict(workspace=_z(64)[::2]), False), (dict(x=x.int()), False), (dict(x=_z(6, 64, dtype=I8)[:, :k - 1]), False), (dict(x=_z(64, 6, dtype=I8).t()[:, :k]), False),
                       (dict(x_scale=_z(5)), False), (dict(x_scale=_z(6, dtype=BF)), False), (dict(out=_z(6, W.outputs).half()), False), (dict(out=_z(5, W.outputs)), False),
                       (dict(out=_z(6, W.outputs + 1)), False)):
        a, b = both(lambda: api.dlm_q8_gemm(**dict(base, **change)))
        assert a == b and both.taken == ok and (type(a) is list) == ok, change
    # the last row's bytes up to a multiple of 16 have to be there
    short = _z(5 * 64 + k, dtype=I8).as_strided((6, k), (64, 1))
    a, b = both(lambda: api.dlm_q8_gemm(**dict(base, x=short)))
    assert a == b and (type(a) is list) == (k % 16 == 0)
    both.status = -3
    assert both(lambda: api.dlm_q8_gemm(**base, workspace=_z(16))) == [api.DlmError, api.DlmError] and both.taken


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """What is built goes to a folder of its own."""
    monkeypatch.setattr(build, "OUT_Q8", str(tmp_path / "_q8.so"))
    return tmp_path


def test_a_build_without_torch_goes_on(monkeypatch, elsewhere, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)  # (an import of it raises ImportError)
    assert build.build_q8_extension() is None and "ctypes" in capsys.readouterr().err
    assert not list(elsewhere.iterdir())


def test_an_extension_of_another_torch_is_not_used(monkeypatch):
    load = api._q8_calls.__wrapped__
    assert load() is not None, "the extension has not been built"
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert load() is None
