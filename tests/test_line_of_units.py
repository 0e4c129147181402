"""How paged_attention's kernel spreads units over blocks: csrc/line.cuh, compiled for the host, against whole numbers of any size."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_13170_b200", "csrc")
SHIM = """#include "line.cuh"
extern "C" long long mul_div(long long a, int b, long long d) { return amph::mul_div(a, b, d); }
extern "C" int block_of(long long u, long long total, int n) { return amph::block_of(u, total, n); }
"""


@pytest.fixture(scope="module")
def line(tmp_path_factory):
    d = tmp_path_factory.mktemp("line")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "line.so")],
                   check=True)
    lib = C.CDLL(str(d / "line.so"))
    lib.mul_div.argtypes, lib.mul_div.restype = [C.c_longlong, C.c_int, C.c_longlong], C.c_longlong
    lib.block_of.argtypes, lib.block_of.restype = [C.c_longlong, C.c_longlong, C.c_int], C.c_int
    return lib


# 4096 sequences of 2^25 + 1 units, 1024 items each: 2^47 and a few more
TOTALS = [1, 2, 63, 64, 1000, 99991, 2 ** 23 - 1, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 1, 2 ** 40 + 12345, 4096 * 1024 * (2 ** 25 + 1)]
# on both sides of a product of 2^32
TOTALS += [2 ** 32 // n + d for n in (2, 148, 444, 592) for d in (-1, 0, 1)]


@pytest.mark.parametrize("n", [1, 2, 3, 7, 148, 444, 592])
def test_borders_and_owners(line, n):
    for total in TOTALS:
        if total < n:
            continue
        borders = [line.mul_div(total, c, n) for c in range(n + 1)]
        assert borders == [total * c // n for c in range(n + 1)] and borders[-1] == total
        for c in range(n):
            for u in {borders[c], borders[c] + 1, (borders[c] + borders[c + 1]) // 2, borders[c + 1] - 1}:
                if borders[c] <= u < borders[c + 1]:
                    assert line.block_of(u, total, n) == c


def test_every_unit_of_a_short_line(line):
    for n in (1, 2, 5, 29, 444):
        for total in (n, n + 1, 2 * n - 1, 3 * n + 2, 4001):
            if total >= n:
                owner = [line.block_of(u, total, n) for u in range(total)]
                assert owner == [c for c in range(n) for _ in range(total * c // n, total * (c + 1) // n)]


def test_items_of_a_sequence(line):
    """mul_div(u, 1, span): the item that a unit of a sequence belongs to."""
    for u in (0, 1, 2 ** 32 - 1, 2 ** 32, 2 ** 47):
        for span in (2, 3, 1024, 2 ** 25 + 1, 2 ** 33):
            assert line.mul_div(u, 1, span) == u // span
