"""How many CTAs of the kernel that keeps rows share an SM (csrc/split_rules.cuh, on the CPU): against a count of what the
SM hands out, for every size a slice can have."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SM, SYSTEM, MOST, BLOCKS = 228 * 1024, 1024, 200 * 1024, 3
SRC = """
#include "split_rules.cuh"
using namespace estp;
extern "C" int room(int sm, int fixed, int n, int most) { return cta_room(sm, fixed, n, most); }
extern "C" int ctas(int64_t bytes, const int* room, int blocks) { return ctas_of(bytes, room, blocks); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(SRC)
    lib = str(d / "rules.so")
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2608_15592_gb300", "csrc"), str(d / "rules.cpp"), "-o", lib], check=True)
    return ctypes.CDLL(lib)


@pytest.mark.parametrize("static", [9344, 9600, 9604, 10000])
def test_ctas_of_every_slice(rules, static):
    fixed = static + SYSTEM
    room = (ctypes.c_int * BLOCKS)(*(rules.room(SM, fixed, n, MOST) for n in range(1, BLOCKS + 1)))
    assert list(room) == sorted(room, reverse=True) and room[0] == MOST
    for n in range(1, BLOCKS + 1):
        assert n * -(-(room[n - 1] + fixed) // 128) * 128 <= SM
    for bytes_ in range(0, MOST + 33, 16):
        holds = [n for n in range(1, BLOCKS + 1) if bytes_ <= MOST and n * -(-(bytes_ + fixed) // 128) * 128 <= SM]
        assert rules.ctas(ctypes.c_int64(bytes_), room, BLOCKS) == max(holds, default=0), bytes_
