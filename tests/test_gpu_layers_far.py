"""The operators around a language model's layers where offsets pass 32 bits, and captured before any other call."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2107_13490_b200 import binding as B  # noqa: E402
from tests import layers_reference as R  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_table_of_more_than_2_to_the_31_elements():
    vocab, dim, n = 550001, 4096, 300
    table = torch.zeros((vocab, dim), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    far = torch.cat([torch.arange(vocab - 200, vocab, device="cuda"), torch.arange(100, device="cuda")])
    table[far] = torch.randn((300, dim), generator=g, device="cuda").bfloat16()
    ids = far[torch.randint(300, (n,), generator=g, device="cuda")]
    assert torch.equal(B.adapt_embedding(table, ids), table[ids])
    dy = torch.randn((n, dim), generator=g, device="cuda").bfloat16()
    del table
    grad = B.adapt_embedding_backward(dy, ids, vocab)
    rows, tol = R.embedding_gradient(dy, torch.searchsorted(far.sort().values, ids), 300, 1.0)
    want = rows[torch.searchsorted(far.sort().values, far)]
    assert R.within(grad[far], want, R.half_step(want, torch.bfloat16) + 1.01 * tol[torch.searchsorted(far.sort().values, far)])
    grad[far] = 0
    assert not grad.any()


def test_rows_of_more_than_2_to_the_31_elements():
    rows, dim = 550001, 4096
    block = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    block[-50:] = torch.randn((50, dim), generator=g, device="cuda").bfloat16()
    w = torch.rand(dim, generator=g, device="cuda") + 0.5
    r = B.adapt_block_norm(block, weight_before=w, want_y=False, want_stats=True)
    small = B.adapt_block_norm(block[-50:].clone(), weight_before=w, want_y=False, want_stats=True)
    assert torch.equal(r.normed[-50:], small.normed) and not r.normed[:-50].any()
    back = B.adapt_block_norm_backward(block, r.stats, d_normed=r.normed, weight_before=w)
    want = B.adapt_block_norm_backward(block[-50:].clone(), small.stats, d_normed=small.normed, weight_before=w)
    assert torch.equal(back.d_block[-50:], want.d_block) and not back.d_block[:-50].any()
    # the sums over rows are taken in another order: 50 terms
    assert torch.allclose(back.d_weight_before, want.d_weight_before, rtol=1e-4, atol=1e-4)


def test_a_product_of_more_than_2_to_the_31_results():
    rows, n, k = 70001, 32768, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randint(-127, 128, (rows, k), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    w = torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    one = torch.ones(1, device="cuda")
    y = B.adapt_int8_linear(x, w, one, x_scales=one, dtype=torch.bfloat16)
    for part in (slice(0, 300), slice(rows - 300, rows)):
        want = (x[part].double() @ w.double().t())
        assert R.within(y[part], want, R.half_step(want, torch.bfloat16))


CAPTURE = r"""
import torch
from paper_2107_13490_b200 import binding as B
torch.cuda.init()
g = torch.Generator(device="cuda").manual_seed(1)
rand = lambda *s: torch.randn(s, generator=g, device="cuda")
table, ids, dy = rand(300, 64), torch.randint(300, (5000,), generator=g, device="cuda"), rand(5000, 64)
x, res, gate, w, d = rand(70, 512), rand(70, 512), rand(70, 512), rand(512), rand(70, 512)
codes = torch.randint(-127, 128, (640, 512), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
scales, many = rand(640), rand(1500, 512)

def calls():
    out = [B.adapt_embedding(table, ids), B.adapt_embedding_backward(dy, ids, 300)]
    r = B.adapt_block_norm(x, residual=res, gate=gate, weight_after=w, weight_before=w, after=B.NORM_RMS, want_stats=True)
    b = B.adapt_block_norm_backward(x, r.stats, d_y=d, d_normed=d, residual=res, gate=gate, weight_after=w, weight_before=w, after=B.NORM_RMS)
    out += [r.y, r.normed, b.d_block, b.d_residual, b.d_gate, b.d_weight_after, b.d_weight_before]
    return out + [B.adapt_int8_linear(v, codes, scales) for v in (x[:1], x, many)]

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    captured = calls()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(captured, calls()))
print("CAPTURED")
"""


def test_the_first_calls_of_a_process_may_be_captured():
    out = subprocess.run([sys.executable, "-c", CAPTURE], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=600)
    assert out.returncode == 0 and "CAPTURED" in out.stdout, out.stdout[-2000:] + out.stderr[-4000:]
