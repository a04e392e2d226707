"""Runs of eight elements of a row and dropout's workgroups for them, on the host, up to the longest rows and the most of them."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LONGEST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("row_plan") / "row_plan.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", os.path.join(HERE, "row_plan_shim.cpp"), "-o", lib], check=True)
    L = C.CDLL(lib)
    L.runs.restype = C.c_uint
    return L


@pytest.mark.parametrize("d", [1, 7, 8, 9, 32768, LONGEST - 8, LONGEST - 7, LONGEST - 6, LONGEST - 1, LONGEST])
def test_runs(L, d):
    assert L.runs(d) == -(-d // 8)


@pytest.mark.parametrize("T", [1, 3, 65536, LONGEST])
@pytest.mark.parametrize("d", [1, 2048, 2049, LONGEST - 7, LONGEST])
def test_workgroups(L, T, d):
    assert L.grid(T, d, 8192) == min(8192, -(-T * -(-d // 8) // 256))
