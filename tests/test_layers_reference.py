"""The 64-bit implementations of the layer operators against differentiation and differences.  CPU only."""
import itertools

import pytest
import torch

from tests import layers_reference as R


def test_embedding_gradient_is_the_transpose():
    g = torch.Generator().manual_seed(1)
    table, dy = torch.randn(7, 5, generator=g).double(), torch.randn(30, 5, generator=g).double()
    ids = torch.randint(-1, 8, (30,), generator=g)
    grad, _ = R.embedding_gradient(dy, ids, 7, 1.5)
    out = R.embedding(table, ids, 1.5)
    live = (ids >= 0) & (ids < 7)
    assert torch.allclose((out[live] * dy[live]).sum(), (grad * table).sum())
    assert (out[ids < 0] == 0).all() and out[ids >= 7].isnan().all()


@pytest.mark.parametrize("after,before,gate,residual", list(itertools.product((0, 1, 2), (0, 1, 2), ("none", "each", "shared"), (False, True))))
def test_norm_gradients_against_differences(after, before, gate, residual):
    g = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    inputs = {"block": rand(4, 9)}
    if residual:
        inputs["residual"] = rand(4, 9)
    if gate != "none":
        inputs["gate"] = rand(9) if gate == "shared" else rand(4, 9)
    if after:
        inputs["weight_after"] = rand(9)
    if before:
        inputs["weight_before"] = rand(9)
    d_y, d_n = rand(4, 9), rand(4, 9) if before else None

    def forward(v, **k):
        return R.Norms(v["block"], v.get("residual"), v.get("gate"), v.get("weight_after"), v.get("weight_before"), after, before,
                       gate == "each", 0.5, 1.25, 1e-5, **k)

    def total(v):
        f = forward(v)
        return (f.y * d_y).sum() + ((f.normed * d_n).sum() if before else 0.0)

    grads = forward(inputs, d_y=d_y, d_normed=d_n)
    for name, v in inputs.items():
        direction, h = rand(*v.shape), 1e-5
        up, down = ({**inputs, name: v + s * h * direction} for s in (1, -1))
        slope = (total(up) - total(down)) / (2 * h)
        # central differences: the third derivative (of order 100 here) by h^2, and 2^-50 of the total by 1 / h
        assert abs(slope - (getattr(grads, "d_" + name) * direction).sum()) <= 1e-7, name


def test_codes():
    x = torch.tensor([[1.0, -2.0, 0.5, 2.0], [0, 0, 0, 0], [1e-35, 0, 0, 0], [float("inf"), 1, 2, 3]])
    codes, scales = R.int8_rows(x)
    assert codes[0].tolist() == [64, -127, 32, 127]      # 63.5 and 31.75: the first to even
    assert (codes[1:] == 0).all()
    assert scales[0] == torch.tensor(2.0) / 127 and scales[1] == scales[2] and scales[3].isnan()
