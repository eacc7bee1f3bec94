"""The operators around a language model's layers on the bounds-checking build of the library: the places of sorted
tokens are table indices that are formed from the data."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

OPERATORS = r"""
import pytest
from paper_2107_13490_b200 import binding as B
checking, word = B.adapt_bounds_check_status(clear=True)
assert checking, "the bounds-checking build was not loaded"
rc = pytest.main(["-q", "-x", "-p", "no:cacheprovider", "tests/test_gpu_embedding.py", "tests/test_gpu_int8.py", "-k", "not extreme_codes"])
assert rc == 0, rc
checking, word = B.adapt_bounds_check_status()
print("BOUNDS", int(checking), *[int(v) for v in word])
"""


def test_no_index_leaves_its_table():
    from paper_2107_13490_b200 import build
    lib = build.build(check=True)
    env = dict(os.environ, ADAPT_B200_LIBRARY=lib, PYTHONPATH=ROOT)
    out = subprocess.run([sys.executable, "-c", OPERATORS], cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    assert out.returncode == 0, out.stdout[-4000:] + out.stderr[-4000:]
    line = [ln for ln in out.stdout.splitlines() if ln.startswith("BOUNDS")][-1].split()
    assert line[1:] == ["1", "0", "0", "0", "0"], line
