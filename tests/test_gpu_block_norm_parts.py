"""Gradients of the norms around a block where only a part of them is asked for or given."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2107_13490_b200 import binding as B  # noqa: E402
from tests.test_gpu_block_norm import EPS, TYPES, check, make  # noqa: E402

NONE, RMS, LAYER = B.NORM_NONE, B.NORM_RMS, B.NORM_LAYER


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("before", [NONE, RMS])
@pytest.mark.parametrize("rows,dim", [(300, 1001), (90, 2047), (70, 4096)])
def test_the_residual_is_not_looked_at_without_the_second_norm_s_gradient(dtype, before, rows, dim):
    """Its values and its place in memory are nothing to the other gradients then: the same bits as without one."""
    v, d_y, _ = make(rows, dim, dtype)
    v["residual"] = v["residual"][:1].expand(rows, dim)      # one row for all: it lies otherwise than the others where dim is odd
    v["weight_before"] = None if before == NONE else v["weight_before"]
    how = dict(after=LAYER, before=before, scale=0.5, residual_scale=1.25, eps=EPS)
    check(v, d_y, None, LAYER, before)
    stats = B.adapt_block_norm(**v, **how, want_stats=True).stats
    got = B.adapt_block_norm_backward(stats=stats, d_y=d_y, **v, **how)
    want = B.adapt_block_norm_backward(stats=stats, d_y=d_y, **{**v, "residual": None}, **how)
    for n in ("d_block", "d_gate", "d_weight_after"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n
    assert want.d_residual is None and got.d_residual.shape == (rows, dim)


def test_the_second_norm_s_weight_has_no_gradient_without_the_output_s():
    v, d_y, d_n = make(40, 256, torch.float32)
    how = dict(after=RMS, before=RMS, eps=EPS)
    stats = B.adapt_block_norm(**v, **how, want_stats=True).stats
    g = B.adapt_block_norm_backward(stats=stats, d_y=d_y, **v, **how)
    assert g.d_weight_before is None and g.d_weight_after is not None
    # what is left out is 0
    assert (B.adapt_block_norm_backward(stats=stats, d_y=d_y, d_normed=torch.zeros_like(d_n), **v, **how).d_weight_before == 0).all()
    none = {n: t[:0] if t.dim() == 2 else t for n, t in v.items()}
    g = B.adapt_block_norm_backward(stats=stats[:0], d_y=d_y[:0], d_normed=d_n[:0], **none, **how)
    assert (g.d_weight_before == 0).all() and (g.d_weight_after == 0).all()
