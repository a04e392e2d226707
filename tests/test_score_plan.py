"""Which kernel a forward call of attention with rules on its scores takes, on the host."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
BY_ROWS, BY_PAIRS, BY_PARTS = range(3)


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("score_plan") / "score_plan.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", os.path.join(HERE, "score_plan_shim.cpp"), "-o", lib], check=True)
    L = C.CDLL(lib)
    L.threads_by_pairs.restype = C.c_longlong
    return L


def test_routes(L):
    assert L.route(1, 8, 8, 17, 4096) == L.route(1, 8, 8, 1, 64) == BY_ROWS
    assert L.route(1, 8, 8, 16, 65) == L.route(256, 1, 1, 1, 1 << 20) == L.route(128, 1, 1, 1, 4096) == BY_PAIRS
    assert L.route(1, 8, 8, 1, 1025) == L.route(128, 1, 1, 1, 4097) == BY_PARTS


@pytest.mark.parametrize("heads", [(32768, 256, 256), (32768, 511, 511), (1 << 14, 512, 512), (65535, 128, 128), (65535, 255, 255)], ids=str)
@pytest.mark.parametrize("Sk", [65, 128, 1 << 14, 1 << 24])
def test_a_launch_by_pairs_has_a_32_bit_number_of_threads(L, heads, Sk):
    """Every size that the entry points admit: up to 2^24 - 64 rows of heads."""
    B, Hq, Hkv = heads
    for b in (B, B - 1):
        few = L.threads_by_pairs(b, Hq, Hkv, 1) < 1 << 32
        assert (L.route(b, Hq, Hkv, 1, Sk) == BY_ROWS) == (not few), b
