"""The library does not depend on what only the Python side's argument checks need."""
import os
import subprocess

import pytest

from paper_2605_01255_b200 import build as acx_build


@pytest.fixture
def commands(tmp_path, monkeypatch):
    """build() with its outputs elsewhere and its compilers replaced: nvcc writes what it is asked for, g++ fails."""
    for name, path in (("OBJ_DIR", "obj"), ("LIB_PATH", "libacx.so"), ("HOST_PATH", "_acx_host.so")):
        monkeypatch.setattr(acx_build, name, str(tmp_path / path))
    ran = []

    def run(cmd, **kw):
        tool = os.path.basename(cmd[0])
        ran.append((tool, cmd[cmd.index("-o") + 1]))
        if "nvcc" in tool:
            open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0 if "nvcc" in tool else 1, "", "no such file: Python.h")

    monkeypatch.setattr(acx_build.subprocess, "run", run)
    return ran


def test_a_host_module_that_cannot_be_built_leaves_the_library(commands):
    with pytest.raises(RuntimeError, match="libacx.so is built; the argument checks") as err:
        acx_build.build()
    assert "Python.h" in str(err.value.__cause__)
    assert os.path.exists(acx_build.LIB_PATH) and not os.path.exists(acx_build.HOST_PATH)
    assert [o for t, o in commands if t != "nvcc"] == [acx_build.HOST_PATH]


def test_no_torch_leaves_the_library(commands, monkeypatch):
    def no_torch(force):
        raise ImportError("No module named 'torch'")

    monkeypatch.setattr(acx_build, "_host_job", no_torch)
    with pytest.raises(RuntimeError, match="libacx.so is built") as err:
        acx_build.build()
    assert isinstance(err.value.__cause__, ImportError) and os.path.exists(acx_build.LIB_PATH)


def test_the_library_alone(commands):
    assert acx_build.build(library_only=True) == acx_build.LIB_PATH
    assert os.path.exists(acx_build.LIB_PATH) and all(t == "nvcc" for t, _ in commands)
