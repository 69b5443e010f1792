"""The build: the C library needs nvcc alone, the torch front end is built beside it where the machine has what that takes."""
import os
import subprocess

import pytest

from paper_2609_21594_b200 import build as b


@pytest.fixture
def machine(monkeypatch, tmp_path):
    """A build into an empty folder whose compilers are stand-ins that write their outputs."""
    ran = []

    def run(cmd, **kw):
        ran.append(os.path.basename(cmd[0]))
        with open(cmd[cmd.index("-o") + 1], "w"):
            pass
        return 0

    class Popen:
        returncode = 0

        def __init__(self, cmd, **kw):
            run(cmd)

        def communicate(self):
            return "", ""

    monkeypatch.setattr(b, "HERE", str(tmp_path))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libmuon_b200.so"))
    monkeypatch.setattr(b, "FRONT", str(tmp_path / "_front.so"))
    monkeypatch.setattr(subprocess, "Popen", Popen)
    monkeypatch.setattr(subprocess, "check_call", run)
    return ran


def test_both_are_built_and_then_nothing(machine):
    assert b.needs_build() and b.build() == b.LIB
    assert machine == ["nvcc"] * (len(b.SOURCES) + 1) + ["g++"]
    machine.clear()
    assert not b.needs_build() and b.build() == b.LIB and not machine


def test_the_library_needs_nvcc_alone(machine, monkeypatch, capsys):
    monkeypatch.setattr(b.shutil, "which", lambda name: None)
    monkeypatch.setattr(b.importlib.util, "find_spec", lambda name: None)
    assert b.front_lacks()[:2] == ["C++ compiler", "torch"]
    assert b.build() == b.LIB and os.path.exists(b.LIB) and not os.path.exists(b.FRONT)
    assert set(machine) == {"nvcc"} and "is not built: no C++ compiler, no torch" in capsys.readouterr().err
    machine.clear()
    b.build()
    assert not machine                                       # the library is there: nothing is compiled again


def test_library_alone_and_each_by_its_own_sources(machine):
    b.build_library()
    assert set(machine) == {"nvcc"} and not os.path.exists(b.FRONT)
    machine.clear()
    b.build()
    assert machine == ["g++"]
    machine.clear()
    later = os.path.getmtime(b.FRONT) - 100
    os.utime(b.FRONT, (later, later))                        # a newer library or front.cpp: the front end again, no kernel
    b.build()
    assert machine == ["g++"]
