"""The library is made also where the Python module over it cannot be; compilers that only write their output stand in for the real ones."""
import builtins
import os
import stat
import subprocess

import pytest

from paper_1911_00472_amd import build


@pytest.fixture
def made(tmp_path, monkeypatch):
    """Sources, results and a compiler for the library in a folder of its own."""
    hipcc = tmp_path / "hipcc"
    hipcc.write_text("#!/bin/sh\nwhile [ $# -gt 0 ]; do if [ \"$1\" = -o ]; then echo made > \"$2\"; fi; shift; done\n")
    hipcc.chmod(hipcc.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("HIPCC", str(hipcc))
    for name in ("SRC", "SRC_TRAIN", "SRC_DISTILL"):
        monkeypatch.setattr(build, name, str(tmp_path / (name + ".hip")))
    monkeypatch.setattr(build, "SRC_BIND", str(tmp_path / "bind.cpp"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libpcr.so"))
    monkeypatch.setattr(build, "MODULE", str(tmp_path / "_train.so"))
    return tmp_path


@pytest.mark.parametrize("compiler", ["false", "/nowhere/a-compiler"])
def test_a_module_that_does_not_compile(made, monkeypatch, compiler):
    monkeypatch.setenv("CXX", compiler)
    (made / "_train.so").write_text("of another library")
    with pytest.raises((subprocess.CalledProcessError, OSError)):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.MODULE)


def test_no_pytorch(made, monkeypatch):
    real = builtins.__import__

    def without(name, *a, **k):
        if name == "torch":
            raise ImportError("no torch")
        return real(name, *a, **k)
    monkeypatch.setattr(builtins, "__import__", without)
    with pytest.raises(ImportError):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.MODULE)


def test_a_library_that_does_not_compile(made, monkeypatch):
    monkeypatch.setenv("HIPCC", "false")
    monkeypatch.setenv("CXX", "true")
    with pytest.raises(subprocess.CalledProcessError):
        build.build()
    assert not os.path.exists(build.LIB) and not os.path.exists(build.MODULE)


def test_both(made, monkeypatch):
    monkeypatch.setenv("CXX", str(made / "hipcc"))
    assert build.build() == build.LIB
    assert os.path.exists(build.LIB) and os.path.exists(build.MODULE)
