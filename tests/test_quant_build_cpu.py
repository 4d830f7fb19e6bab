"""The build where something of torch is not there, and a module that was built for another torch (no GPU needed)."""

import os
import sys

import pytest
import torch

from paper_2602_01901_b200 import build as qbuild
from paper_2602_01901_b200 import quant


@pytest.fixture
def built(monkeypatch):
    """The tree as it is built; what a test builds of the extension is only counted."""
    qbuild.build()
    made = []
    monkeypatch.setattr(qbuild, "_build_extension", lambda: made.append(1))
    return made


def test_what_is_built_stays(built):
    assert qbuild.build() == qbuild.LIB and not built


def test_another_torch_builds_the_module_again(built, monkeypatch):
    monkeypatch.setattr(torch, "__version__", "1.0.0+other")
    qbuild.build()
    assert built == [1]


def test_another_python_builds_the_module_again(built, monkeypatch):
    monkeypatch.setattr(sys, "version_info", (3, 99, 0, "final", 0))
    assert qbuild._extension_is_stale()


def test_a_newer_source_builds_the_module_again(built, monkeypatch):
    source = os.path.join(qbuild.CSRC, "qc_torch.cpp")
    older, there = qbuild._older, qbuild.EXTENSION
    monkeypatch.setattr(qbuild, "_older", lambda target, sources: target == there and "qc_torch.cpp" in sources or older(target, sources))
    assert os.path.exists(source)
    qbuild.build()
    assert built == [1]


def test_without_torch_the_library_is_built_alone(built, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)      # import torch raises
    assert qbuild.build() == qbuild.LIB and qbuild.build(force=False) == qbuild.LIB
    assert not built and "quant.py" in capsys.readouterr().err


def test_without_headers_the_library_is_built_alone(built, monkeypatch, capsys):
    import sysconfig

    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": "/nowhere"})
    assert qbuild.build() == qbuild.LIB
    assert not built and "Python.h" in capsys.readouterr().err


def test_a_module_for_another_torch_is_not_used(built, monkeypatch):
    monkeypatch.setattr(quant, "_calls", None)
    monkeypatch.setattr(torch, "__version__", "1.0.0+other")
    with pytest.raises(RuntimeError, match="1.0.0.other.*build it again"):
        quant._native()
