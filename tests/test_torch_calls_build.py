"""Which compiled module of csrc/dkv_torch.cpp is loaded: that of these sources, or none."""
import os
import shutil
import sysconfig

import pytest

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


def test_no_sources_no_module(sources):
    os.remove(sources / "dkv_torch.cpp")
    assert dkv._torch_calls("1.2") is None
