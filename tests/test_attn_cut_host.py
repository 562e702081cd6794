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
int longest_item(unsigned long long steps, int heads, int places, int min_steps) { return ssm::longest_item(steps, heads, places, min_steps); }
int cut_tile(int steps, int most, int* len) {
    const auto c = ssm::cut_tile(steps, most);
    *len = c.len;
    return c.pieces;
}
int item_bin(int len, int most, int bins) { return ssm::item_bin(len, most, bins); }
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


def _cut(cut, steps, most):
    n = ctypes.c_int()
    return cut.cut_tile(steps, most, ctypes.byref(n)), n.value


@pytest.mark.parametrize("rows,heads,kv_heads,cached", [(1 << 18, 32, 1, 1 << 30), (1 << 22, 128, 128, 1 << 30), (1 << 22, 128, 1, 1 << 30),
                                                        (1 << 22, 1, 1, 1 << 30)])
@pytest.mark.parametrize("places", [256, 512])
def test_items_at_the_limits_of_a_call(cut, rows, heads, kv_heads, cached, places):
    """All rows behind the longest cache: more steps than 32 bits count. No tile is cut there, and every item has a bin."""
    tiles = rows * (heads // kv_heads) // 128
    each = cached // 64 + 1
    cut.longest_item.argtypes = [ctypes.c_ulonglong, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    most = cut.longest_item(tiles * each, kv_heads, places, 8)
    assert most >= min(each, -(-tiles * each * kv_heads // places))
    for grown in (most, most + most * 15 // 16, (most + 1) // 2):
        for steps in (0, 1, 8, each - 1, each):
            pieces, n = _cut(cut, steps, grown)
            assert pieces >= 1 and n <= max(grown, 0) and (pieces - 1) * n < max(steps, 1) <= max(pieces * n, 1)
            assert 0 <= cut.item_bin(n, grown, 32) < 32


def test_items_of_ordinary_calls(cut):
    cut.longest_item.argtypes = [ctypes.c_ulonglong, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    assert cut.longest_item(0, 8, 512, 8) == 8
    assert cut.longest_item(1000, 8, 512, 8) == 16 and cut.longest_item(1000, 8, 512, 2) == 16
    assert _cut(cut, 9, 8) == (2, 5) and _cut(cut, 8, 8) == (1, 8) and _cut(cut, 69, 14) == (5, 14) and _cut(cut, 0, 8) == (1, 0)
    assert _cut(cut, 3, 2) == (2, 2)
    for most in (1, 2, 8, 100):
        bins = [cut.item_bin(n, most, 32) for n in range(most + 1)]
        assert bins == sorted(bins, reverse=True) and bins[0] == 31 and bins[-1] >= 0
