"""What is built when: the library needs no PyTorch, and the extension module is that of one PyTorch version."""
import os

import pytest

torch = pytest.importorskip("torch")
from paper_1712_01084_b200 import binding as pb
from paper_1712_01084_b200 import build as pbuild


def test_the_library_builds_without_the_extension_module(monkeypatch):
    def refuse(*args, **kw):
        raise AssertionError("the extension module is not part of the library")
    monkeypatch.setattr(pbuild, "build_torch", refuse)
    monkeypatch.setattr(pbuild, "needs_build", lambda: False)
    assert pbuild.build() == pbuild.LIB


def test_the_module_of_another_torch_is_not_fresh(monkeypatch, tmp_path):
    pbuild.build_torch()
    assert not pbuild.needs_build_torch()
    monkeypatch.setattr(torch, "__version__", torch.__version__ + "1")
    assert pbuild.needs_build_torch()
    other = tmp_path / "_pp_torch.so"
    monkeypatch.setattr(pbuild, "TORCH_LIB", str(other))
    assert pbuild.needs_build_torch()                                        # missing
    other.write_bytes(b"..made for torch " + torch.__version__.encode() + b"\0..")
    assert not pbuild.needs_build_torch()
    os.utime(other, (1, 1))
    assert pbuild.needs_build_torch()                                        # older than its sources


def test_the_module_of_another_torch_is_not_loaded(monkeypatch):
    pb._load_torch()
    monkeypatch.setattr(torch, "__version__", "1.0")
    with pytest.raises(ImportError, match="build it again"):
        pb._load_torch()
