"""The token embedding's gradient added to a given one: widths that are read element by element, gradients that begin between
16-byte boundaries, and so many tokens that frequent ones are cut and joined."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2107_13490_b200 import binding as B  # noqa: E402
from tests import layers_reference as R  # noqa: E402
from tests.test_gpu_embedding import draw_ids, rand  # noqa: E402


@pytest.mark.parametrize("dtype,grad", [(torch.float32, torch.float32), (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16),
                                        (torch.float16, torch.float32), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("how", ["even", "one", "few", "wild"])
@pytest.mark.parametrize("n,vocab,dim,at", [(500, 60, 33, 0), (3000, 700, 1001, 0), (5000, 100, 48, 1), (20011, 3000, 7, 0), (65537, 513, 40, 8),
                                            (40000, 2, 1, 3)])
def test_is_the_sum(dtype, grad, how, n, vocab, dim, at):
    ids, dy = draw_ids(n, vocab, how), rand(n, dim, dtype=dtype)
    buf = rand(vocab, dim + 9, seed=5, dtype=grad)
    start, beside = buf[:, at:at + dim].clone(), buf.clone()
    got = B.adapt_embedding_backward(dy, ids, vocab, scale=0.75, dtable=buf[:, at:at + dim], accumulate=True)
    assert got.data_ptr() == buf[:, at:].data_ptr()
    want, tol = R.embedding_gradient(dy, ids, vocab, 0.75)
    want = want + start.double()
    # the sum's own bound, one more addition, the rounding to the type
    assert R.within(got, want, R.half_step(want, grad) + 1.01 * tol + R.U * want.abs())
    absent = torch.ones(vocab, dtype=torch.bool, device="cuda")
    absent[ids[(ids >= 0) & (ids < vocab)]] = False
    assert torch.equal(got[absent], start[absent])
    assert torch.equal(buf[:, :at], beside[:, :at]) and torch.equal(buf[:, at + dim:], beside[:, at + dim:])
    again = beside[:, at:at + dim]
    assert torch.equal(B.adapt_embedding_backward(dy, ids, vocab, scale=0.75, dtable=again, accumulate=True), got)
