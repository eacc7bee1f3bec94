"""How rows of the norms around a block are dealt to threads and CTAs (csrc/norm_shape.h): every length fits the CTAs of a
cluster and the places that their sums have, wherever the row begins.  Compiled with g++; nothing runs on a GPU."""
import os
import subprocess

from paper_2107_13490_b200 import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2107_13490_b200", "csrc")
SOURCE = """
#include <cstdio>
#include "../../include/adapt.h"
#include "norm_shape.h"
using namespace adapt;
#define NEED(c) if (!(c)) { std::printf("%s: dim %d, %d elements of %d threads, %d parts\\n", #c, dim, s.elems, s.threads, s.parts); return 1; }
int check(int dim, const NormShape& s, int most, int parts) {
  NEED(s.threads >= 32 && s.threads % 32 == 0 && s.threads <= most)
  NEED(s.parts >= 1 && s.parts <= parts)
  NEED(s.per_sm >= 1)
  const int in_front = dim % 8 ? 7 : 0, width = s.elems * s.threads;
  NEED(in_front + dim <= width * s.parts)
  NEED(in_front + dim > width * (s.parts - 1))   // no part without elements
  return 0;
}
int main() {
  for (int dim = 1; dim <= ADAPT_NORM_MAX_DIM; ++dim) {
    if (check(dim, norm_forward(dim), kNormMaxThreads, kNormMaxParts)) return 1;
    if (check(dim, norm_backward(dim), kNormBackwardThreads, kNormMaxParts)) return 1;
    for (int norms = 1; norms <= 2; ++norms)
      if (norm_in_pairs(dim, norms) && check(dim, norm_backward_pairs(dim), kNormPairThreads, 1)) return 1;
  }
}
"""


def test_every_length_fits(tmp_path):
    (tmp_path / "norm_shape.cpp").write_text(SOURCE.replace("../../include", os.path.join(CSRC, "../../include")))
    program = str(tmp_path / "norm_shape")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(tmp_path / "norm_shape.cpp"), "-o", program], check=True)
    r = subprocess.run([program], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


def test_long_rows_have_sums_of_a_cta_on_every_sm():
    """Rows that lie otherwise go to CTAs of which each takes a whole row: no fewer than there are SMs (148)."""
    for dim in (1, 8, 333, 1000, 4096, 8192, 8193, 9000, 16384, 16385, 20001, B.NORM_MAX_DIM):
        assert B.adapt_block_norm_workspace_bytes(100000, dim) >= 3 * 4 * 148 * dim, dim
        assert B.adapt_block_norm_workspace_bytes(3, dim) >= 3 * 4 * 3 * dim, dim
