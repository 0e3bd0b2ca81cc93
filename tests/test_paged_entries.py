"""What an append takes of the caller's lengths and starts (csrc/paged.h compiled by the host compiler): all of a
sequence's new rows or none, by the rules of uad_kv_append, whichever kernel looks at them."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_37772_amd", "csrc")

SRC = r"""
#include "%s/paged.h"
using namespace uad;
extern "C" {
int take(int b, int from, int to, int rows, int len, int pages, int shift) { return sequence_ok(b, from, to, rows, len, pages, shift); }
int length(int len, int pages, int shift, int *bad) { bool x = false; int n = length_or_none(len, pages, shift, &x); *bad = x; return n; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("entries")
    (d / "p.cpp").write_text(SRC % CSRC)
    subprocess.run(["g++", "-O1", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", str(d / "p.cpp"), "-o", str(d / "p.so")], check=True)
    return ctypes.CDLL(str(d / "p.so"))


@pytest.mark.parametrize("length,pages,shift,want", [(0, 1, 4, 0), (16, 1, 4, 16), (17, 1, 4, None), (-1, 1, 4, None), (2 ** 31 - 1, 1, 8, None),
                                                     (-2 ** 31, 9, 4, None), (2 ** 30, 2 ** 22, 8, 2 ** 30), (2 ** 30 + 1, 2 ** 22, 8, None)])
def test_a_length_that_cannot_be_used_counts_as_none(lib, length, pages, shift, want):
    bad = ctypes.c_int()
    assert lib.length(length, pages, shift, ctypes.byref(bad)) == (want or 0) and bad.value == (want is None)


def refused(lib, starts, lens, rows, pages=4, shift=4):
    return [b for b in range(len(lens)) if not lib.take(b, starts[b], starts[b + 1], rows, lens[b], pages, shift)]


@pytest.mark.parametrize("starts,lens,rows,want", [
    ([0, 3, 5], [3, 2], 3, [1]),                       # rows that do not exist
    ([0, 3, 5, 4], [3, 2, 0], 3, [1, 2]),
    ([0, 2, 1, 2, 2, 1], [40] * 5, 2, [1, 4]),         # falls, though every row has one sequence that could take it
    ([0, 0, 2], [-1, 2], 2, [0]),                      # lengths of sequences without rows
    ([0, 0, 2], [65, 64], 2, [0]),
    ([0, 0, 0], [0, 64], 0, []),
    ([1, 2, 3], [9, 9], 3, [0]),
    ([0, 64, 65], [64, 1], 65, []),
    ([0, 64, 65], [63, 1], 65, [0]),
    ([0, 2 ** 31 - 1], [64], 2 ** 31 - 1, [0]),
    ([0, -2 ** 31, 2 ** 31 - 1], [64, 64], 2 ** 31 - 1, [0, 1]),
])
def test_sequences_that_are_refused(lib, starts, lens, rows, want):
    assert refused(lib, starts, lens, rows) == want


def test_starts_and_lengths_pass_as_they_are_defined(lib):
    r = np.random.default_rng(6)
    seen = [0, 0]
    for _ in range(4000):
        n, rows = int(r.integers(1, 6)), int(r.integers(0, 7))
        starts = [0] + sorted(int(x) for x in r.integers(0, rows + 1, n))
        if r.random() < 0.5:
            starts[int(r.integers(0, n + 1))] = int(r.integers(-1, rows + 3))
        lens = [int(x) for x in r.integers(0, 67, n)] if r.random() < 0.5 else [64] * n
        fine = (starts[0] == 0 and all(0 <= a <= b <= rows for a, b in zip(starts, starts[1:]))
                and all(b - a <= m <= 64 for a, b, m in zip(starts, starts[1:], lens)))
        assert (refused(lib, starts, lens, rows) == []) == fine, (starts, lens, rows)
        seen[fine] += 1
    assert min(seen) > 400
