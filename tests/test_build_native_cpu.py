"""The build without what only the Python binding needs: the C libraries are linked whether or not the extension module can be built, and
a module for another Python or torch is not taken."""
import os
import sys
import sysconfig

import pytest
import torch

import paper_2604_23108_amd as M
from paper_2604_23108_amd import block_binding as B
from paper_2604_23108_amd import build


@pytest.fixture
def linked(monkeypatch):
    """The build's steps without the compiler; which libraries were linked."""
    out = []
    monkeypatch.setattr(build, "_compile", lambda src: src)
    monkeypatch.setattr(build, "_link", lambda lib, objs, extra=(): out.append(lib))
    return out


def test_libraries_are_linked_where_the_module_does_not_compile(linked, monkeypatch):
    def fails(*_):
        raise RuntimeError("no headers")
    monkeypatch.setattr(build, "_native", fails)
    with pytest.raises(RuntimeError, match="no headers"):
        build.build()
    assert linked == [build.LIB, build.BENCH_LIB]


def test_without_torch_there_are_the_libraries_alone(linked, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)              # import torch raises ImportError
    assert build.build() == build.LIB
    assert linked == [build.LIB, build.BENCH_LIB]
    assert "torch" in capsys.readouterr().err


def test_the_module_belongs_to_this_python_and_torch():
    name = os.path.basename(build.native_path(torch.__version__))
    assert name.startswith("_block_native.") and name.endswith(".so")
    assert sysconfig.get_config_var("SOABI") in name and torch.__version__ in name
    B._native.rmsnorm
    assert B._native.file == build.native_path(torch.__version__)


def test_a_module_for_another_torch_is_not_loaded(monkeypatch):
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    with pytest.raises(M.MohgeError, match="0.0.1.* is missing: build it"):
        B._Native().rmsnorm


def test_names_that_the_module_lacks_are_attribute_errors():
    with pytest.raises(AttributeError, match="no_such_call"):
        B._native.no_such_call
    assert not hasattr(B._native, "__wrapped__")
