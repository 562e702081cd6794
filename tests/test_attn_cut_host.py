"""The prompt attention's plan arithmetic (csrc/attn_cut.h) compiled for the host, at the limits of a call."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_21144_amd", "csrc")
SOURCE = """
#include "attn_cut.h"
extern "C" {
int tiles_of_rows(int m, int heads, int rows) { return ssm::tiles_of_rows(m, heads, rows); }
int add_tiles(int a, int b) { return ssm::add_tiles(a, b); }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    d = tmp_path_factory.mktemp("cut")
    (d / "cut.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", "-Wall", "-Werror", "-I" + CSRC, str(d / "cut.cpp"),
                    "-o", str(d / "cut.so")], check=True)
    return ctypes.CDLL(str(d / "cut.so"))


def test_sums_of_overlapping_sequences_stay_in_order(cut):
    most = cut.tiles_of_rows(1 << 22, 128, 128)
    assert most == 1 << 22
    at, last = 0, -1
    for _ in range(1 << 14):   # every second of 2^15 sequences claims all rows of the largest call
        at = cut.add_tiles(at, most)
        assert at >= last and at >= 0
        last = at
    assert at > (1 << 22) + (1 << 15)      # seen to be more than any call has
    assert cut.add_tiles(at, at) == at and cut.add_tiles(at, 0) == at


def test_sums_of_a_call_are_exact(cut):
    assert cut.add_tiles(0, 0) == 0 and cut.add_tiles(12345, 678) == 13023
    assert cut.add_tiles(1 << 22, 1 << 15) == (1 << 22) + (1 << 15)
    for m, g, rows in ((0, 8, 128), (1, 1, 128), (128, 1, 128), (129, 1, 128), (1 << 22, 128, 256), (33, 4, 128)):
        assert cut.tiles_of_rows(m, g, rows) == -(-m * g // rows)
