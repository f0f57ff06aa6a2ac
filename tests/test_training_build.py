"""How the build goes about the module of the training calls: after the C library, which needs none of its headers; again for another torch; and
left out, loudly, where it cannot be compiled."""
import subprocess
import sysconfig
from pathlib import Path

import pytest
import torch

from paper_2609_31975_b200 import build, training


@pytest.fixture()
def place(monkeypatch, tmp_path):
    """The module and its stamp in a folder of their own, and a compiler that only writes its output file and keeps its commands."""
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        Path(cmd[cmd.index("-o") + 1]).write_bytes(b"module")
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build, "CALLS", tmp_path / "_training.so")
    monkeypatch.setattr(build, "OBJ", tmp_path / "build")
    monkeypatch.setattr(build.subprocess, "run", run)
    return tmp_path, ran


def test_the_library_comes_first(monkeypatch):
    steps = []
    monkeypatch.setattr(build, "build_library", lambda *a: steps.append("library") or Path("lib"))

    def broken(force):
        steps.append("module")
        raise RuntimeError("no headers")

    monkeypatch.setattr(build, "build_calls", broken)
    with pytest.raises(RuntimeError, match="no headers"):
        build.build()
    assert steps == ["library", "module"]


def test_it_is_built_again_for_another_torch(place, monkeypatch):
    _, ran = place
    assert build.build_calls() == build.CALLS and len(ran) == 1
    build.build_calls()
    assert len(ran) == 1                                   # nothing has changed
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    build.build_calls()
    assert len(ran) == 2 and '-DSFFN_TORCH="9.9.9"' in ran[1]
    build.build_calls()
    assert len(ran) == 2


@pytest.mark.parametrize("lacking", ["headers", "compiler"])
def test_it_is_left_out_where_it_cannot_be_compiled(place, monkeypatch, lacking):
    folder, ran = place
    build.CALLS.write_bytes(b"older module")               # of a build that no stamp vouches for
    if lacking == "headers":
        monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": str(folder / "nowhere")})
    else:
        monkeypatch.setenv("CXX", "a-compiler-that-is-not-there")
    with pytest.warns(UserWarning, match="training calls"):
        assert build.build_calls() is None
    assert not ran and not build.CALLS.exists()


def test_a_module_for_another_torch_is_not_used(monkeypatch):
    build.build()
    monkeypatch.setattr(training, "_bound", None)
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    with pytest.raises(RuntimeError, match="was built for torch"):
        training._calls()
