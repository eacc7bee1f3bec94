"""The pieces in which a dropout call is launched cover its rows and columns exactly once, whatever the sizes.
Host arithmetic (csrc/dropout_pieces.h), compiled with g++; nothing runs on a GPU."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2107_13490_b200", "csrc")
SOURCE = """
#include "dropout_pieces.h"
extern "C" long long pieces(long long rows, long long cols, int unit, long long most, long long* out) {
  long long n = 0;
  const adapt::DropoutPieces all(rows, cols, unit);
  all.each([&](int64_t r, int64_t c, int64_t nr, int64_t nc) {
    if (n == most) return 1;
    long long* at = out + 5 * n++;
    at[0] = r; at[1] = c; at[2] = nr; at[3] = nc; at[4] = all.per_row * nr;
    return 0;
  });
  return n;
}
"""


@pytest.fixture(scope="module")
def pieces(tmp_path_factory):
    where = tmp_path_factory.mktemp("pieces")
    (where / "pieces.cpp").write_text(SOURCE)
    lib = str(where / "pieces.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC,
                    str(where / "pieces.cpp"), "-o", lib], check=True)
    f = ctypes.CDLL(lib).pieces
    f.restype = ctypes.c_longlong
    f.argtypes = [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_void_p]

    def run(rows, cols, unit):
        out = np.zeros((1 << 18, 5), dtype=np.int64)
        n = f(rows, cols, unit, len(out), out.ctypes.data)
        assert n < len(out)
        return [tuple(int(v) for v in p) for p in out[:n]]

    return run


@pytest.mark.parametrize("unit", [8, 4, 2])     # elements of a chunk: 16-bit, fp32, pairs
def test_pieces_cover_every_element_once(pieces, unit):
    cap = unit * ((1 << 27) - 1)                # elements of the longest row that one launch takes
    sizes = [(1, 1), (1, cap + 9), (3, 7), (1 << 20, 10), (1 << 34, 3), (5000, 1 << 20)]
    for cols in (cap - 1, cap, cap + 1, cap + 8, 2 * cap, 2 * cap + 5, 1_200_000_000, (1 << 31) - 1, 1 << 31, (1 << 33) + 3):
        sizes += [(rows, cols) for rows in (1, 2, 8, 9, 1000)]
    for rows, cols in sizes:
        at_row, at_col = 0, 0       # what is still to come begins here
        for row, col, n_rows, n_cols, chunks in pieces(rows, cols, unit):
            assert (row, col) == (at_row, at_col), (rows, cols)
            assert n_rows >= 1 and n_cols >= 1 and row + n_rows <= rows and col + n_cols <= cols
            # several rows together are whole rows: the kernel walks each of them from end to end
            assert n_rows == 1 or (col == 0 and n_cols == cols), (rows, cols, row, col, n_rows, n_cols)
            assert n_rows == 1 or (n_cols < 1 << 31 and chunks < 1 << 31)
            assert col % unit == 0      # the pieces of a row meet at whole chunks
            if col + n_cols == cols:
                at_row, at_col = row + n_rows, 0
            else:
                at_row, at_col = row, col + n_cols
        assert (at_row, at_col) == (rows, 0), (rows, cols)
