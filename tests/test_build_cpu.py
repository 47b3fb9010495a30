"""When the compiled argument marshalling is built; the compiler is replaced by a record."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2604_17397_b200 import build


@pytest.fixture
def runs(monkeypatch, tmp_path):
    """Commands that would have been run, for a binding of its own in an empty folder."""
    done = []
    monkeypatch.setattr(build, "BINDING_PATH", str(tmp_path / "_binding.so"))

    def run(cmd, check):
        done.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w"):
            pass

    monkeypatch.setattr(subprocess, "run", run)
    return done


def test_the_binding_is_built_once_and_again_for_another_torch(runs, monkeypatch):
    assert build.build_binding() == build.BINDING_PATH and len(runs) == 1
    build.build_binding()
    assert len(runs) == 1                               # as it is
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    build.build_binding()
    build.build_binding()
    assert len(runs) == 2                               # for the other torch, once
    monkeypatch.undo()


def test_the_binding_is_built_again_when_its_source_is_newer(runs):
    build.build_binding()
    os.utime(build.BINDING_PATH, (1, 1))
    build.build_binding()
    assert len(runs) == 2
    build.build_binding(force=True)
    assert len(runs) == 3


def test_a_build_that_failed_is_not_taken_for_one(runs, monkeypatch):
    build.build_binding()

    def fail(cmd, check):
        raise subprocess.CalledProcessError(1, cmd)

    with monkeypatch.context() as m:
        m.setattr(subprocess, "run", fail)
        m.setattr(torch, "__version__", "0.0.1")
        for _ in range(2):
            with pytest.raises(subprocess.CalledProcessError):
                build.build_binding()
    build.build_binding()                               # the first one is still in place, and right for this torch
    assert len(runs) == 1


def test_the_library_alone_builds_without_torch(runs, monkeypatch, tmp_path):
    monkeypatch.setitem(sys.modules, "torch", None)
    lib = str(tmp_path / "libsdvg.so")
    monkeypatch.setattr(build, "LIB_PATH", lib)
    assert build.build(out=lib) == lib
    assert [c[c.index("-o") + 1] for c in runs] == [lib]
    assert build.build(out=lib) == lib and len(runs) == 1
