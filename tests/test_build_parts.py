"""The simulator's library builds with hipcc alone; the iteration operators' binding needs more and says so."""
import os

import pytest

from paper_2602_02987_amd import build


@pytest.fixture
def commands(monkeypatch):
    """build() without compiling: the commands it would run."""
    ran = []
    monkeypatch.setattr(build, "_compile", lambda src, force, verbose: src + ".o")
    monkeypatch.setattr(build.subprocess, "check_call", lambda cmd: ran.append(cmd))
    return ran


def _outputs(commands):
    return [c[c.index("-o") + 1] for c in commands]


def test_library_and_binding(commands):
    build.build()
    assert _outputs(commands) == [build.LIB, build.BINDING]


def test_without_torch(commands, monkeypatch, capfd):
    import importlib.util
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert build.build() == build.LIB and _outputs(commands) == [build.LIB]
    assert "torch" in capfd.readouterr().err


def test_without_pythons_headers(commands, monkeypatch, capfd, tmp_path):
    import sysconfig
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **kw: dict(include=str(tmp_path)))
    build.build()
    assert _outputs(commands) == [build.LIB] and "Python.h" in capfd.readouterr().err


def test_without_a_host_compiler(commands, monkeypatch, capfd):
    monkeypatch.setenv("CXX", "/no/such/compiler")
    build.build()
    assert _outputs(commands) == [build.LIB] and "/no/such/compiler" in capfd.readouterr().err


def test_a_binding_that_does_not_compile_is_an_error(commands, monkeypatch):
    def fails(*a):
        raise build.subprocess.CalledProcessError(1, "g++")
    monkeypatch.setattr(build, "build_binding", fails)
    with pytest.raises(build.subprocess.CalledProcessError):
        build.build()
    assert os.path.basename(build.BINDING) == "_iteration.so"
