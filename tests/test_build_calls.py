"""The build of the direct calls (csrc/layer_calls.cpp): one module per Python and torch,
and a failed compile is not repeated."""
import os
import subprocess

import pytest
import torch

from paper_2505_12728_gb300 import build_lib
from paper_2505_12728_gb300 import specflash_verify as sfv


@pytest.fixture
def place(tmp_path, monkeypatch):
    """An empty build folder, and the g++ runs that build_calls makes."""
    runs = []
    real = subprocess.run

    def run(cmd, **kw):
        runs.append(cmd)
        return real(cmd, **kw)

    monkeypatch.setattr(build_lib, "BUILD", str(tmp_path))
    monkeypatch.setattr(build_lib.subprocess, "run", run)
    return tmp_path, runs


def trivial(tmp_path, monkeypatch, text="int specflash_nothing;\n"):
    """A source that compiles in no time (or not at all)."""
    src = tmp_path / "calls.cpp"
    src.write_text(text)
    os.utime(src, (0, 0))
    monkeypatch.setattr(build_lib, "CALLS_SOURCE", str(src))


def test_another_torch_gets_a_module_of_its_own(place, monkeypatch):
    tmp_path, runs = place
    trivial(tmp_path, monkeypatch)
    first = build_lib.build_calls()
    assert first and os.path.exists(first) and len(runs) == 1
    assert build_lib.build_calls() == first and len(runs) == 1  # up to date
    monkeypatch.setattr(torch, "__version__", "9.9.9+other")
    second = build_lib.build_calls()
    assert second != first and os.path.exists(second) and len(runs) == 2
    monkeypatch.setattr(build_lib.sysconfig, "get_config_var", lambda name: "cpython-999-any")
    assert build_lib.calls_path() not in (first, second)


def test_a_module_of_another_torch_is_not_loaded(place, monkeypatch):
    tmp_path, runs = place
    trivial(tmp_path, monkeypatch)
    build_lib.build_calls()
    monkeypatch.setattr(torch, "__version__", "9.9.9+other")
    monkeypatch.setattr(sfv, "_calls", None)

    def no_load(*a):
        raise AssertionError("a module of another torch was looked at")

    monkeypatch.setattr(sfv.importlib.util, "spec_from_file_location", no_load)
    sfv._load_calls(None)
    assert sfv._calls is None


def test_a_failed_compile_is_not_repeated(place, monkeypatch, capsys):
    tmp_path, runs = place
    trivial(tmp_path, monkeypatch, "this is no C++\n")
    assert build_lib.build_calls() is None and len(runs) == 1
    assert "not built" in capsys.readouterr().err
    assert build_lib.build_calls() is None and len(runs) == 1
    assert build_lib.build_calls(force=True) is None and len(runs) == 2
    trivial(tmp_path, monkeypatch)  # mended
    os.utime(build_lib.CALLS_SOURCE)
    for name in os.listdir(tmp_path):
        if name.endswith(".failed"):
            os.utime(tmp_path / name, (1, 1))
    assert build_lib.build_calls() and len(runs) == 3
