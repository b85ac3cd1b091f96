"""Which rows the paged cache's kernels touch in a ragged call: their own arithmetic (csrc/sage_paged_rows.h), compiled for the CPU.  The threads of a
workgroup look at all sequences, and whoever finds the workgroup's tile in its sequence writes five numbers for the others: with row
starts that are not ascending several can, and each number is then one of theirs, in any mixture."""
import ctypes
import itertools
import os
import subprocess

import pytest

from tile_copy import CSRC

SOURCE = """
#include "sage_paged_rows.h"
extern "C" {
int claim(int a, int b, int i, int T, int rows, int per, int x, int *out) {
    const sage::RowClaim c = sage::row_claim(a, b, i, T, rows, per);
    out[0] = x - c.first, out[1] = c.q0, out[2] = c.q1 - c.q0;
    return sage::claims(c, x);
}
int rows_left(int q0, int n, int T) { return sage::rows_left(q0, n, T); }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_rows")
    src, out = str(d / "rows.cpp"), str(d / "rows.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
    return ctypes.CDLL(out)


def _claims(lib, starts, T, rows, per, x):
    """(tile, first row, rows) of every sequence that claims tile x."""
    out, got = (ctypes.c_int * 3)(), []
    for i in range(len(starts) - 1):
        if lib.claim(starts[i], starts[i + 1], i, T, rows, per, x, out):
            got.append(tuple(out))
    return got


def _grid(T, B, rows, per):
    return T * per // rows + B


@pytest.mark.parametrize("rows,per", [(64, 1), (64, 4), (128, 3), (8, 4)])
def test_starts_of_all_kinds_stay_within_the_calls_rows(lib, rows, per):
    T = 1000
    passed = 0
    for starts in ([0, T, 5, T - 3, 0, T], [T, 0, T, 1], [400, 900, 300, 800, 200, 1 << 30, -5, T], [0, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], [0, T] * 40):
        for x in range(_grid(T, len(starts) - 1, rows, per)):
            found = _claims(lib, starts, T, rows, per, x)
            assert all(tile >= 0 for tile, _, _ in found)
            for q0, n in itertools.product({q0 for _, q0, _ in found}, {n for _, _, n in found}):
                passed += q0 + n > T                      # what the numbers of two sequences can say
                left = lib.rows_left(q0, n, T)
                assert 0 <= q0 < T and 0 < left <= n and q0 + left <= T
    assert passed > 0


@pytest.mark.parametrize("rows,per", [(64, 1), (64, 8), (192, 5), (16, 1)])
def test_ascending_starts_give_every_tile_one_sequence(lib, rows, per):
    for T, starts in ((1000, [0, 1, 1, 65, 500, 999, 1000]), (7, [2, 3, 3, 7]), (4000, [0, 4000]), (300, list(range(0, 301, 3)))):
        covered = [0] * T
        for x in range(_grid(T, len(starts) - 1, rows, per)):
            found = _claims(lib, starts, T, rows, per, x)
            assert len(found) <= 1
            for tile, q0, n in found:
                assert lib.rows_left(q0, n, T) == n
                for r in range(tile * rows, min((tile + 1) * rows, n * per)):
                    covered[q0 + r // per] += 1
        assert covered == [per if starts[0] <= t < starts[-1] else 0 for t in range(T)]
