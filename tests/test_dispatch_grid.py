"""Grids of more workgroups than a launch takes along one axis (csrc/agc_dispatch.h), compiled with the host compiler.  The
embedding's gradient has such ones: 2^26 tokens of 2000 values are 2^24 workgroups of 256 threads.  CPU only."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DRIVER = r"""
#include "agc_dispatch.h"
extern "C" void grid(int64_t workgroups, int threads, unsigned* out)
{
    const agc::FoldedGrid g = agc::folded_grid(workgroups, threads);
    out[0] = g.x, out[1] = g.y;
}
"""


@pytest.fixture(scope="module")
def grid(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("grid")
    (tmp / "driver.cpp").write_text(DRIVER)
    cxx = shutil.which("g++") or shutil.which("c++")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fPIC", "-shared",
                    "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-I", os.path.join(ROOT, "paper_2605_15890_amd", "csrc"), str(tmp / "driver.cpp"),
                    "-o", str(tmp / "libgrid.so")], check=True)
    lib = ctypes.CDLL(str(tmp / "libgrid.so"))
    lib.grid.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_void_p]

    def call(workgroups, threads):
        out = (ctypes.c_uint * 2)()
        lib.grid(workgroups, threads, out)
        return out[0], out[1]

    return call


@pytest.mark.parametrize("workgroups", [1, 2, 1000003, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, 2 ** 25 + 3, 2 ** 29 + 2 ** 23])
@pytest.mark.parametrize("threads", [64, 256, 512])
def test_folded_grid(grid, workgroups, threads):
    x, y = grid(workgroups, threads)
    assert x * threads < 2 ** 32 and y < 65536
    assert workgroups <= x * y < workgroups + y          # as many as are needed, and ids stay below 2^32
    assert y == 1 or workgroups * threads >= 2 ** 32
