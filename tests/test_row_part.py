"""How rows of logits are dealt to CTAs (csrc/row_part.h): every element once, at every alignment, up to the longest
vocabulary; compiled with g++ and its overflow checks.  Nothing runs on a GPU."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2107_13490_b200", "csrc")
SOURCE = """
#include <cstdio>
#include <initializer_list>
#include "row_part.h"
using adapt::RowRange;
#define NEED(c) if (!(c)) { std::printf("%s: count %d mis %d vocab %d rank %d of %d\\n", #c, count, mis, vocab, rank, parts); return 1; }
int check(int count, int mis, int vocab, int parts) {
  long long next = 0, seen = 0;   // the element behind the chunks so far, elements met
  int tail_from = 0, head = 0;
  for (int rank = 0; rank < parts; ++rank) {
    const RowRange r(count, mis, vocab, rank, parts);
    NEED(0 <= r.q0 && r.q0 <= r.q1)
    if (rank == 0) {
      head = r.head; tail_from = r.tail_from; next = head;
      NEED(0 <= r.edges && r.edges <= 2 * (count - 1))
      for (int i = 0; i < r.edges; ++i) {
        const int j = r.edge(i);
        NEED(0 <= j && j < vocab && (j < head || j >= tail_from))
        if (i) NEED(r.edge(i - 1) < j)
        const int q = r.chunk(j);
        for (int other = 0; other < parts; ++other) {   // no part holds it in a chunk
          const RowRange o(count, mis, vocab, other, parts);
          NEED(q < o.q0 || q >= o.q1)
        }
      }
      seen = r.edges;
    } else {
      NEED(r.edges == 0)
    }
    if (r.q0 < r.q1) {
      NEED(r.element(r.q0) == next)
      const long long last = static_cast<long long>(r.element(r.q1 - 1)) + count - 1;
      NEED(last < vocab)
      NEED(r.chunk(r.element(r.q0)) == r.q0 && r.chunk(static_cast<int>(last)) == r.q1 - 1)
      next = last + 1;
      seen += static_cast<long long>(r.q1 - r.q0) * count;
    }
    if (rank == parts - 1) NEED(seen == vocab && (next == tail_from || tail_from >= vocab || next == head))
  }
  return 0;
}
int main() {
  for (int count = 4; count <= 8; count += 4)
    for (int mis = 0; mis < count; ++mis)
      for (int parts = 1; parts <= 16; parts *= 2) {
        for (int vocab = 1; vocab < 300; ++vocab) if (check(count, mis, vocab, parts)) return 1;
        for (int less = 0; less < 20; ++less) if (check(count, mis, 0x7FFFFFFF - less, parts)) return 1;
        for (int vocab : {131072, 50257, 1 << 30}) if (check(count, mis, vocab, parts)) return 1;
      }
}
"""


def test_every_element_once(tmp_path):
    (tmp_path / "row_part.cpp").write_text(SOURCE)
    program = str(tmp_path / "row_part")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC,
                    str(tmp_path / "row_part.cpp"), "-o", program], check=True)
    r = subprocess.run([program], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
