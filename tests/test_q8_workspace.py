"""dlm_q8_gemm without a workspace: the call takes what its own launch needs, no more, and asks for no other's plan (CPU; nothing is launched)."""
import ctypes as C

import pytest
import torch

from paper_2604_15750_amd import api

VP, I32, I64 = C.c_void_p, C.c_int, C.c_int64
GEMM = C.CFUNCTYPE(I32, VP, VP, I64, VP, I32, VP, I64, I32, VP, C.c_size_t, VP)


def _weight(n, k, gated=False):
    """A Q8Weight without its packed memory."""
    w = object.__new__(api.Q8Weight)
    w.n, w.k, w.gated = n, k, gated
    w._data = torch.zeros(16, dtype=torch.uint8)
    w._desc = api.dlm_q8_weight(n, k, int(gated), w._data.data_ptr())
    w._ref = C.addressof(w._desc)
    return w


@pytest.fixture(params=["extension", "ctypes"])
def calls(request, monkeypatch):
    """calls.seen: (workspace, its bytes) of each C call; calls.taken: what the C calls that were not refused had.  The real planner says what
    a call needs, and no call but Q8Weight.workspace may look through fewer rows."""
    L = api.lib()
    ext = api._q8_calls()
    assert ext is not None, "the extension has not been built"

    class Calls:
        seen, taken = [], []

    def gemm(w, x, x_stride, x_scale, rows, out, out_stride, dtype, ws, size, stream):
        d = C.cast(w, C.POINTER(api.dlm_q8_weight)).contents
        plan = (C.c_int32 * 6)()
        Calls.seen.append((ws, size))
        if x_stride <= 1 << 22:
            if L.dlm_plan_q8_gemm(rows, d.n, d.k, d.gated, plan):
                return -3
            if plan[5] and (not ws or size < plan[5] << 10):
                return -3
        Calls.taken.append((ws, size))
        return 0

    def search(*a):
        raise AssertionError("the plans of fewer rows were looked through")

    entry = GEMM(gemm)

    class Library:
        dlm_q8_gemm, dlm_q8_gemm_workspace = entry, staticmethod(search)
        dlm_plan_q8_gemm, dlm_last_error = L.dlm_plan_q8_gemm, L.dlm_last_error

    Calls.seen, Calls.taken = [], []
    Calls.through_extension = request.param == "extension"
    for name, value in (("lib", lambda: Library), ("_device", lambda: -1), ("_stream", lambda: 0), ("_gpu_of", lambda name, t: -1),
                        ("_q8_calls", (lambda: ext) if Calls.through_extension else (lambda: None))):
        monkeypatch.setattr(api, name, value)
    real = [C.cast(f, VP).value for f in (L.dlm_q8_rows, L.dlm_add_norm_q8, L.dlm_q8_gemm)]
    ext.bind(*real[:2], C.cast(entry, VP).value)
    yield Calls
    ext.bind(*real)


# (rows, n, k): split and not, among them one that needs none where fewer rows need 63 MiB, and one that needs less than fewer rows do
@pytest.mark.parametrize("rows,n,k", [(8, 4096, 256), (64, 512, 8192), (486, 4096, 12288), (2822, 384, 4096), (2822, 512, 16000), (2822, 3584, 18944)])
@pytest.mark.parametrize("given", [False, True])
def test_a_call_takes_its_own_need(calls, rows, n, k, given):
    need = api.plan_q8_gemm(rows, n, k)["workspace_kib"] << 10
    w, x, s = _weight(n, k), torch.zeros(rows, k, dtype=torch.int8), torch.zeros(rows)
    out = torch.zeros(rows, n) if given else None
    got = api.dlm_q8_gemm(w, x, s, out=out, dtype=torch.float32)
    assert got.shape == (rows, n) and (out is None or got is out)
    assert [size for _, size in calls.taken] == [need] and bool(calls.taken[0][0]) == bool(need)
    assert len(calls.seen) <= (2 if need else 1)  # (one that was refused for want of a workspace, and the one that had it)


def test_the_cases_are_what_they_are_for():
    f, plan = api.lib().dlm_q8_gemm_workspace, lambda *a: api.plan_q8_gemm(*a)["workspace_kib"] << 10
    assert plan(2822, 3584, 18944) == 0 and f(2822, 3584, 18944, 0) > 60 << 20
    assert 0 < plan(486, 4096, 12288) < f(486, 4096, 12288, 0) and plan(64, 512, 8192) > 0 and plan(8, 4096, 256) == 0


def test_rows_far_apart_need_none(calls):
    """(They are streamed, whatever their number; as columns of rows 2^22 + 16 bytes long, of which no byte is read.)"""
    rows, n, k = 64, 512, 8192
    memory = torch.empty((rows - 1) * ((1 << 22) + 16) + k, dtype=torch.int8)
    api.dlm_q8_gemm(_weight(n, k), memory.as_strided((rows, k), ((1 << 22) + 16, 1)), torch.zeros(rows), out=torch.zeros(rows, n))
    assert calls.seen == calls.taken == [(None, 0)]


def test_a_call_that_is_too_large_is_still_refused(calls):
    rows = (1 << 20) + 1
    with pytest.raises(api.DlmError, match="ECAPACITY"):
        api.dlm_q8_gemm(_weight(4, 16), torch.zeros(rows, 16, dtype=torch.int8), torch.zeros(rows), dtype=torch.float32)
    assert not calls.taken


def test_a_workspace_that_is_too_small_is_refused(calls):
    """... where it is given: nothing is allocated in its place."""
    rows, n, k = 64, 512, 8192
    with pytest.raises(api.DlmError, match="ECAPACITY"):
        api.dlm_q8_gemm(_weight(n, k), torch.zeros(rows, k, dtype=torch.int8), torch.zeros(rows), out=torch.zeros(rows, n), workspace=torch.zeros(16))
    assert not calls.taken and len(calls.seen) == 1
