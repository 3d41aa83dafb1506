"""Launch sizes that the library computes on the host, built with g++ and tried up to sizes that no test allocates."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_04084_amd", "csrc")

SHIM = """
#include "ld_grid.h"
extern "C" {
int32_t workgroups(int64_t wanted, int32_t threads, int64_t others) { return ld_workgroups(wanted, threads, others); }
int32_t few_clearing(int64_t V, int32_t adding) { return ld_few_clearing(V, adding); }
int32_t clip_grid(int32_t pieces, int32_t in_place) { return ld_clip_grid(pieces, in_place != 0); }
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("grid")
    src, lib = str(d / "shim.cpp"), str(d / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC,
                    src, "-o", lib], check=True)
    return ctypes.CDLL(lib)


def test_workgroups_stay_below_2_32_threads(shim):
    for threads in (64, 256, 512, 1024):
        for others in (0, 1, 8192):
            most = (2 ** 32 - 1) // threads - others
            for wanted in (0, 1, 1000, most - 1, most, most + 1, 2 ** 40):
                got = shim.workgroups(ctypes.c_int64(wanted), threads, ctypes.c_int64(others))
                assert got == min(wanted, most) and (got + others) * threads < 2 ** 32, (threads, others, wanted)


def test_rows_cleared_beside_few_tokens(shim):
    """268.4 M rows and more ask for as many workgroups as a launch has, besides those that add."""
    at = 64 * 4194303
    for V in (1, 63, 64, 65, 70_000_001, at - 64, at, at + 1, 268_435_456, 268_435_457, 2 ** 30, 2 ** 31 - 2):
        for adding in (1, 2, 32, 8192):
            got = shim.few_clearing(ctypes.c_int64(V), adding)
            assert 1 <= got <= (V + 63) // 64 and (got + adding) * 1024 < 2 ** 32, (V, adding)
            assert got == (V + 63) // 64 or (got + adding + 1) * 1024 >= 2 ** 32, (V, adding)


def test_workgroups_that_clip(shim):
    """2^41 elements in all are 2^29 pieces, and one more for each tensor: they are shared out where a launch has no workgroup for each."""
    for pieces in (1, 7, 8, 9, 16384, 16385, 2 ** 24 - 9, 2 ** 24 - 8, 2 ** 24 - 7, 2 ** 24, 2 ** 24 + 1, 2 ** 29 + 2 ** 20):
        places = (pieces + 7) // 8 * 8
        out, inside = shim.clip_grid(pieces, 0), shim.clip_grid(pieces, 1)
        assert out % 8 == 0 and out == min(places, 2 ** 24 - 8) and out * 256 < 2 ** 32, pieces
        assert inside == (places if pieces <= 16384 else 16384), pieces
        assert places - 1 + out < 2 ** 31  # a workgroup's pieces, from one to the next
