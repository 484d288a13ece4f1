"""Workspaces of the operators around a block and at the two ends of the backward pass, and the build, without a GPU."""
import builtins
import ctypes
import os
import subprocess

import pytest

from paper_2205_05632_b200 import build as builder
from paper_2205_05632_b200 import load_library


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return load_library()


@pytest.mark.parametrize("kinds", [(1, 1), (2, 2), (0, 0), (1, 0), (2, 0)], ids=str)
@pytest.mark.parametrize("n,rows,h,vocab", [(8, 1024, 4096, 100000), (8, 1024, 4096, 99999), (1, 1, 4096, 32000), (3, 7, 64, 100), (2, 30000, 64, 20000),
                                            (1, 300, 16384, 1000000), (16, 5, 2048, 50257), (4, 100, 512, 8000), (1, 4, 6144, 777)])
def test_a_head_workspace_for_copies_has_room_without_them(lib, n, rows, h, vocab, kinds):
    def need(shared, x_copied, weight_copied, wanted):
        b = ctypes.c_size_t(0)
        assert lib.compams_head_workspace_bytes(ctypes.byref(b), n, rows, h, vocab, *kinds, shared, x_copied, weight_copied, wanted) == 0
        return b.value

    for shared in (0, 1):
        for wanted in range(4):
            least = [need(shared, x, w, wanted) for x in (0, 1) for w in (0, 1)]
            assert need(shared, 1, 1, wanted) == max(least)
            assert need(shared, 0, 1, wanted) >= need(shared, 0, 0, wanted) and need(shared, 1, 0, wanted) >= need(shared, 0, 0, wanted)


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """Builds into an empty folder with compilers that write their output's name; the commands, and a set of compilers that fail."""
    ran, broken = [], set()

    def run(cmd, check):
        name = os.path.basename(cmd[0])
        ran.append(name)
        if name in broken:
            raise subprocess.CalledProcessError(1, cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built")

    monkeypatch.setattr(builder, "subprocess", type("S", (), {"run": staticmethod(run)}))
    monkeypatch.setattr(builder, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(builder, "EXTENSION", str(tmp_path / "ops.so"))
    monkeypatch.setenv("NVCC", "nvcc")
    monkeypatch.setenv("CXX", "g++")
    return ran, broken


def test_the_library_is_built_without_the_extension(compilers, monkeypatch):
    ran, broken = compilers
    broken.add("g++")
    with pytest.raises(subprocess.CalledProcessError):
        builder.build()
    assert ran == ["nvcc", "g++"] and os.path.exists(builder.LIB) and not os.path.exists(builder.EXTENSION)
    ran.clear()
    known = builtins.__import__

    def without_torch(name, *args, **kw):
        if name == "torch":
            raise ImportError(name)
        return known(name, *args, **kw)

    monkeypatch.setattr(builtins, "__import__", without_torch)
    assert builder.build(force=True) == builder.LIB and ran == ["nvcc"]


def test_the_extension_is_built_for_the_torch_and_the_python_that_are_there(compilers, monkeypatch):
    import sysconfig

    import torch
    ran, _ = compilers
    builder.build()
    assert ran == ["nvcc", "g++"]
    builder.build()
    assert ran == ["nvcc", "g++"]  # nothing has changed
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    builder.build()
    assert ran == ["nvcc", "g++", "g++"]
    monkeypatch.setattr(sysconfig, "get_config_var", lambda name: "cpython-999")
    builder.build()
    builder.build()
    assert ran == ["nvcc", "g++", "g++", "g++"]
