"""The module of the short calls is built beside the library, which is there without it."""
from __future__ import annotations

import os
import subprocess

import pytest

from paper_2607_20538_gb300 import build


class Tools:
    """Stand-ins for the compilers: nvcc leaves an empty file, g++ does as `gxx` says."""

    def __init__(self, gxx):
        self.gxx = gxx

    def run(self, cmd, **kw):
        if cmd[0] == "g++":
            return self.gxx(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")

    def check_call(self, cmd, **kw):
        return self.run(cmd).returncode


def _no_compiler(cmd):
    raise FileNotFoundError(2, "No such file or directory", "g++")


def _fails(cmd):
    return subprocess.CompletedProcess(cmd, 1, "", "python_variable.h:1: needs a later standard")


@pytest.fixture
def place(tmp_path, monkeypatch):
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path / "_build"))
    monkeypatch.setattr(build, "nvcc", lambda: "nvcc")
    open(build.CALLS, "w").close()     # of an earlier build
    os.utime(build.CALLS, (1, 1))
    return tmp_path


@pytest.mark.parametrize("gxx,says", [(_no_compiler, "g++"), (_fails, "needs a later standard")])
def test_the_library_without_the_calls(gxx, says, place, monkeypatch, capsys):
    headers = os.path.join(os.path.dirname(build.importlib.util.find_spec("torch").origin), "include/torch/csrc/autograd/python_variable.h")
    if not (os.path.exists(headers) and os.path.exists(os.path.join(build.sysconfig.get_path("include"), "Python.h"))):
        pytest.skip("no headers to build the module with")
    tools = Tools(gxx)
    monkeypatch.setattr(build.subprocess, "run", tools.run)
    monkeypatch.setattr(build.subprocess, "check_call", tools.check_call)
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert not os.path.exists(build.CALLS)           # nothing made for other sources is left to be loaded
    err = capsys.readouterr().err
    assert says in err and "ctypes" in err


def test_the_library_without_headers(place, monkeypatch, capsys):
    tools = Tools(_no_compiler)
    monkeypatch.setattr(build.subprocess, "run", tools.run)
    monkeypatch.setattr(build.subprocess, "check_call", tools.check_call)
    monkeypatch.setattr(build.sysconfig, "get_path", lambda name: str(place))
    assert build.build() == build.LIB and os.path.exists(build.LIB) and not os.path.exists(build.CALLS)
    assert "Python.h" in capsys.readouterr().err


def test_a_kernel_that_does_not_compile_still_ends_the_build(place, monkeypatch):
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: subprocess.CompletedProcess(cmd, 1, "", "error"))
    with pytest.raises(RuntimeError, match="nvcc"):
        build.build()
