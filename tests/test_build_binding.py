"""What the build asks for: hipcc for the library; torch's and Python's headers for the
binding's module of native checks alone."""
import os
import sys
import sysconfig

import pytest

from paper_2004_11250_amd import build, train


@pytest.fixture
def commands(monkeypatch, tmp_path):
    ran = []

    def run(cmd):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return ""

    monkeypatch.setattr(build, "_run", run)
    monkeypatch.setattr(build, "TENSORS_LIB", str(tmp_path / "_tensors.so"))
    return ran


def test_the_module_is_built_by_hipcc(commands):
    pytest.importorskip("torch")
    assert build.build_tensors() == build.TENSORS_LIB and os.path.exists(build.TENSORS_LIB)
    assert [cmd[0] for cmd in commands] == [build.HIPCC]


@pytest.mark.parametrize("missing", ["torch", "Python.h"])
def test_without_its_headers_it_is_left_out(commands, monkeypatch, tmp_path, capsys, missing):
    if missing == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": str(tmp_path / "none")})
    open(build.TENSORS_LIB, "w").close()        # (one of an earlier build must not stay)
    assert build.build_tensors() is None and not commands and not os.path.exists(build.TENSORS_LIB)
    assert missing in capsys.readouterr().err


def test_calls_that_need_it_say_so(monkeypatch):
    monkeypatch.setitem(sys.modules, "paper_2004_11250_amd._tensors", None)
    monkeypatch.delattr(sys.modules["paper_2004_11250_amd"], "_tensors", raising=False)
    train._native.cache_clear()
    try:
        with pytest.raises(RuntimeError, match="not built"):
            train._native()
    finally:
        train._native.cache_clear()
