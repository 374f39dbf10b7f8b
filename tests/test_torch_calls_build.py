"""Which compiled module of csrc/dkv_torch.cpp is loaded, and what becomes of one that cannot be built or does not load: dkv.py's own
calls go on without it."""
import os
import shutil
import sysconfig

import pytest
import torch

from paper_2609_32663_gb300 import build, dkv


@pytest.fixture
def sources(monkeypatch, tmp_path):
    """The header and the source as copies, and the module beside them."""
    os.makedirs(tmp_path / "include")
    shutil.copy(os.path.join(build.INCLUDE, "dkv.h"), tmp_path / "include" / "dkv.h")
    shutil.copy(os.path.join(build.CSRC, "dkv_torch.cpp"), tmp_path / "dkv_torch.cpp")
    monkeypatch.setattr(build, "INCLUDE", str(tmp_path / "include"))
    monkeypatch.setattr(build, "TORCH_CALLS", str(tmp_path / "dkv_torch.cpp"))
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    monkeypatch.setattr(build, "PKG", str(tmp_path))
    monkeypatch.setattr(build, "OBJDIR", str(tmp_path / "_build"))
    return tmp_path


def compiler(path, monkeypatch, script):
    """A g++ that does this, first on the path (None: no g++ at all)."""
    os.makedirs(path)
    if script is not None:
        (path / "g++").write_text("#!/bin/sh\n" + script)
        os.chmod(path / "g++", 0o755)
    monkeypatch.setenv("PATH", str(path))


@pytest.mark.parametrize("name", ["include/dkv.h", "dkv_torch.cpp"])
def test_other_sources_are_another_module(sources, name):
    """A module that was built from another header or source is not the one that is looked for."""
    first = build.torch_calls("1.2")
    assert build.torch_calls("1.2") == first != build.torch_calls("1.3")
    with open(first, "w") as f:  # (it would not load)
        f.write("a module of the sources as they were")
    with open(sources / name, "a") as f:
        f.write("// and more\n")
    assert build.torch_calls("1.2") != first
    assert dkv._torch_calls("1.2") is None


def test_another_python_is_another_module(sources, monkeypatch):
    first = build.torch_calls("1.2")
    get = sysconfig.get_config_var
    monkeypatch.setattr(sysconfig, "get_config_var", lambda name: "cpython-399-none" if name == "SOABI" else get(name))
    assert build.torch_calls("1.2") != first


def test_a_module_that_does_not_load_is_left_out(sources):
    with open(build.torch_calls("1.2"), "w") as f:
        f.write("no module")
    with pytest.warns(UserWarning, match="does not load"):
        assert dkv._torch_calls("1.2") is None


def test_no_sources_no_module(sources):
    os.remove(sources / "dkv_torch.cpp")
    assert dkv._torch_calls("1.2") is None


@pytest.mark.parametrize("script", ["echo no >&2; exit 1\n", None])
def test_a_build_that_fails_is_told_and_is_no_error(sources, monkeypatch, tmp_path, script):
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        pytest.skip("no headers of Python")
    compiler(tmp_path / "bin", monkeypatch, script)
    with pytest.warns(UserWarning, match="g\\+\\+"):
        assert build.build_torch_calls() is None
    assert dkv._torch_calls(torch.__version__) is None


def test_it_is_built_where_it_can_be():
    """(A source that does not compile is not to pass for a missing compiler.)"""
    if shutil.which("g++") is None or not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        pytest.skip("no g++ or no headers of Python")
    assert build.build_torch_calls() == build.torch_calls(torch.__version__)
    assert dkv._torch_calls(torch.__version__).quant_attn
