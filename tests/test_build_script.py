"""What the build script builds and when, with the compilers replaced by a recorder."""
import os
import sys

import pytest

from paper_2011_05630_amd import build as B


@pytest.fixture
def built(tmp_path, monkeypatch):
    """-> the compilers called; what they build are empty files in a folder of the test's own."""
    calls = []

    def run(cmd, target, tmp):
        calls.append(os.path.basename(cmd[0]))
        with open(target, "w") as f:
            f.write(" ".join(cmd))
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libdlf.so"))
    monkeypatch.setattr(B, "TORCH_LIB", str(tmp_path / "_dlf_torch.so"))
    monkeypatch.setattr(B, "_run", run)
    return calls


def test_both_by_default(built):
    assert B.needs_build() and B.needs_build_torch()
    assert B.build() == B.LIB
    assert built == ["hipcc", "g++"]
    assert not B.needs_build() and not B.needs_build_torch()
    B.build(force=False)
    assert built == ["hipcc", "g++"]
    B.build()
    assert built == ["hipcc", "g++"] * 2


def test_the_c_library_alone(built):
    """A program of the C calls needs neither PyTorch's headers nor g++."""
    B.build(library_only=True)
    assert built == ["hipcc"] and not B.needs_build() and B.needs_build_torch()
    B.build(force=False, library_only=True)
    assert built == ["hipcc"]


def test_without_pytorch(built, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    B.build()
    assert built == ["hipcc"] and "PyTorch" in capsys.readouterr().out


def test_another_pytorch(built, monkeypatch):
    """The module is built against one PyTorch and belongs to it."""
    import torch
    B.build()
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert B.needs_build_torch() and not B.needs_build()
    B.build(force=False)
    assert built == ["hipcc", "g++", "g++"]
    assert not B.needs_build_torch()


def test_older_than_their_sources(built):
    B.build()
    old = min(os.path.getmtime(os.path.join(B.CSRC, f)) for f in B.SOURCES + B.HEADERS + [B.TORCH_SOURCE]) - 10
    os.utime(B.TORCH_LIB, (old, old))
    assert B.needs_build_torch() and not B.needs_build()
    os.utime(B.LIB, (old, old))
    assert B.needs_build()


def test_a_module_of_another_pytorch_says_so(monkeypatch):
    import torch
    from paper_2011_05630_amd import feedforward as F
    F._native()
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    with pytest.raises(RuntimeError, match="0.0.1"):
        F._native()


def test_a_missing_module_says_so(monkeypatch):
    from paper_2011_05630_amd import feedforward as F
    monkeypatch.setitem(sys.modules, "paper_2011_05630_amd._dlf_torch", None)
    monkeypatch.delattr("paper_2011_05630_amd._dlf_torch", raising=False)
    with pytest.raises(RuntimeError, match="not built"):
        F._native()
