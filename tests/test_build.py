"""What building the library needs, and what it leaves where torch's headers or g++ are missing (nothing is compiled here)."""
import os
import subprocess

import pytest

from paper_2603_12118_amd import binding as B
from paper_2603_12118_amd import build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        return subprocess.CompletedProcess(cmd, 1 if cmd[0] == "g++" else 0, "", "no torch/csrc/autograd/python_variable.h")
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    return ran


def test_the_library_needs_hipcc_alone(commands):
    assert build.build_library() == build.LIB
    assert len(commands) == len(build.SOURCES) + 1 and {cmd[0] for cmd in commands} == {"hipcc"}


def test_calls_that_do_not_compile_are_an_error_and_leave_no_old_ones(commands):
    open(build.CALLS, "w").close()
    with pytest.raises(RuntimeError, match=r"calls.cpp:\nno torch/csrc"):
        build.build_calls()
    assert not os.path.exists(build.CALLS)


def test_the_library_runs_without_them(monkeypatch):
    monkeypatch.setattr(B, "_calls_module", None)
    import builtins
    real = builtins.__import__

    def without(name, globals=None, locals=None, fromlist=(), level=0):
        if level and "_calls" in (fromlist or ()):
            raise ImportError("_calls")
        return real(name, globals, locals, fromlist, level)
    monkeypatch.setattr(builtins, "__import__", without)
    assert B.cs_cache_query(2, 128, 32)[0] == 2 * 32 * 136           # ctypes
    import torch
    x = torch.zeros(4, 2, 128)
    with pytest.raises(RuntimeError, match="_calls.so is not built"):
        B.cs_cache_write(x, x, x, x, 32)
