"""The extension behind the 8-bit cache's Python calls is optional: where it cannot be built, or was built against another torch, they go through ctypes."""
import sys

import pytest
import torch

from paper_2604_15750_amd import api, build


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
