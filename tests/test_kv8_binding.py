"""The extension behind the 8-bit cache's Python calls is optional: where it cannot be built, or was built against another torch, they go through ctypes."""
import sys

import pytest
import torch

from paper_2604_15750_amd import api, build
from test_kv8_host import both, cpu_cache  # noqa: F401


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """What is built goes to a folder of its own."""
    monkeypatch.setattr(build, "OUT_KV8", str(tmp_path / "_kv8.so"))
    return tmp_path


def test_a_build_without_torch_goes_on(monkeypatch, elsewhere, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)  # (an import of it raises ImportError)
    assert build.build_kv8_extension() is None and "ctypes" in capsys.readouterr().err
    assert not list(elsewhere.iterdir())


def test_a_build_that_the_compiler_refuses_goes_on(monkeypatch, elsewhere, capsys):
    (elsewhere / "torch").mkdir()
    monkeypatch.setattr(torch, "__file__", str(elsewhere / "torch" / "__init__.py"))  # (no headers there)
    assert build.build_kv8_extension() is None
    assert "kv8_py.cpp" in (err := capsys.readouterr().err) and "ctypes" in err


def test_an_extension_of_another_torch_is_not_used(monkeypatch):
    load = api._kv8_calls.__wrapped__
    assert load() is not None, "the extension has not been built"
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert load() is None


def test_calls_ask_torch_for_the_device(monkeypatch):
    """torch initialises its side of the GPU there, and refuses a process forked from one that had: no call goes past it, whether it has a tensor or not."""
    monkeypatch.setattr(api, "_raw_stream", lambda dev: ("stream of", dev))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 5)
    assert api._stream() == ("stream of", 5) and api._device() == 5

    def refused():
        raise RuntimeError("Cannot re-initialize CUDA in forked subprocess")

    monkeypatch.setattr(torch.cuda, "current_device", refused)
    x, pos = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32)
    cache = api.Kv8Cache(2, 64, 2, 64, device="cpu")
    for call in (api.probe_mfma, lambda: api.dlm_kv8_write(cache, x, x, [0, 4], [0]), lambda: api.dlm_kv8_read(cache, [0, 4], [0], k=x, v=x),
                 lambda: api.dlm_kv8_attention(cache, x, [0, 4], [4], out=x), lambda: api.dlm_qk_norm_rope(x[:, 0], pos, 1, 0, 64, out=x[:, 1])):
        with pytest.raises(RuntimeError, match="forked"):
            call()


@pytest.mark.parametrize("rows", [1, 2])
def test_views_of_one_row_are_taken_as_those_of_several(both, rows):
    """A row has no stride: in place into fewer columns, or from a number of columns that is no multiple of 16 bytes, is the same call for any number of rows."""
    wide = torch.zeros(rows, 408)
    pos = torch.zeros(rows, dtype=torch.int32)
    for x, out in ((wide[:, :400], wide[:, :192]), (wide[:, :193], wide[:, :400]), (wide[:, :401], torch.zeros(rows, 200)[:, :195]), (wide, wide)):
        a, b = both(lambda: api.dlm_qk_norm_rope(x, pos, 2, 1, 64, out=out))
        assert a == b and both.taken
        x_stride, out_stride = a[0][1], a[0][13]
        assert x_stride % 4 == 0 and out_stride % 4 == 0 and x_stride >= 192 and out_stride >= 192
        assert x_stride == out_stride or x.data_ptr() != out.data_ptr()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_row_in_place(device, dtype):
    wide = torch.randn(2, 408, device=device).to(dtype)
    pos = torch.tensor([7, 7], dtype=torch.int32, device=device)
    gain = torch.full((64,), 1.5, device=device).to(dtype)
    want = api.dlm_qk_norm_rope(wide[:, :193], pos, 2, 1, 64, gain, gain)
    for rows in (2, 1):
        x = wide.clone()
        api.dlm_qk_norm_rope(x[:rows, :401], pos[:rows], 2, 1, 64, gain, gain, out=x[:rows, :193])
        assert torch.equal(x[:rows, :192], want[:rows]) and torch.equal(x[:rows, 192:], wide[:rows, 192:]) and torch.equal(x[rows:], wide[rows:])


def test_sizes_below_32_bits():
    """They would arrive at the library as their low 32 bits."""
    for bad in ((1 - 2**32, 64, 2, 64), (1, 64 - 2**32, 2, 64), (1, 64, 2 - 2**32, 64), (1, 64, 2, 64 - 2**32), (-1, 64, 2, 64)):
        with pytest.raises(api.DlmError, match="ESHAPE"):
            api.Kv8Cache(*bad, device="cpu")


def test_a_workspace_that_is_not_contiguous_is_refused_either_way(both, cpu_cache):
    q, out = torch.zeros(6, 4, 64), torch.zeros(6, 4, 64)
    for ws, ok in ((torch.zeros(64, dtype=torch.uint8), True), (torch.zeros(128, dtype=torch.uint8)[::2], False), (torch.zeros(16, 4).t(), False)):
        a, b = both(lambda: api.dlm_kv8_attention(cpu_cache, q, [0, 6], [9], out=out, workspace=ws))
        assert a == b and both.taken == ok and (a is ValueError) != ok
