"""The library builds with no torch, and beside one without CUDA: the binding of its operators is then left out."""

import importlib.util
import os

from paper_1811_12843_gb300 import _build


def test_the_binding_needs_a_torch_with_cuda(tmp_path, monkeypatch):
    torch = tmp_path / "torch"
    (torch / "lib").mkdir(parents=True)
    (torch / "__init__.py").write_text("")
    found = importlib.util.spec_from_file_location("torch", str(torch / "__init__.py"))
    monkeypatch.setattr(importlib.util, "find_spec", lambda name: found)
    assert _build._torch_dir() is None
    (torch / "lib" / "libc10_cuda.so").write_text("")
    assert _build._torch_dir() == os.path.dirname(found.origin)
    monkeypatch.setattr(importlib.util, "find_spec", lambda name: None)
    assert _build._torch_dir() is None
