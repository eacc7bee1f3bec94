"""Norms around a block over long rows: those that the CTAs of a cluster share, at the lengths where the room in front of an
odd row tips it into another shape, and over so many rows that a cluster's ring of stages and the places of its sums are used
in turn many times."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2107_13490_b200 import binding as B  # noqa: E402
from tests.test_gpu_block_norm import TYPES, check, make  # noqa: E402

NONE, RMS, LAYER = B.NORM_NONE, B.NORM_RMS, B.NORM_LAYER


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("rows,dim", [(3, 8185), (3, 8186), (3, 8191), (3, 16378), (3, 16383), (2, 32761), (2, 32762), (2, 32764), (2, 32767), (2, 32768)])
def test_lengths_at_the_borders_of_shapes(dtype, kind, rows, dim):
    v, d_y, d_n = make(rows, dim, dtype)
    check(v, d_y, d_n, kind, kind)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("after,before,gate", [(RMS, LAYER, "each"), (LAYER, NONE, "shared"), (NONE, RMS, "none")])
@pytest.mark.parametrize("rows,dim", [(400, 7168), (301, 12288), (301, 20001), (151, 32762), (151, 32764), (151, 32767), (151, 32768)])
def test_many_long_rows(dtype, after, before, gate, rows, dim):
    v, d_y, d_n = make(rows, dim, dtype, gate)
    check(v, d_y, d_n, after, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate", ["each", "shared"])
@pytest.mark.parametrize("rows,dim", [(1300, 1024), (700, 4096), (613, 9000), (451, 16384), (301, 20001), (151, 32768)])
def test_many_rows_that_lie_otherwise(dtype, gate, rows, dim):
    """The residual begins behind the other tensors' 16-byte boundaries; CTAs take several rows each."""
    v, d_y, d_n = make(rows, dim, dtype, gate)
    buf = torch.zeros((rows, dim + 8), dtype=dtype, device="cuda")
    buf[:, 1:1 + dim] = v["residual"]
    v["residual"] = buf[:, 1:1 + dim]
    check(v, d_y, d_n, RMS, LAYER)
