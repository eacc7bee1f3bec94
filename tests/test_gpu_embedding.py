"""Token embedding and its gradient against their definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2107_13490_b200 import binding as B  # noqa: E402
from tests import layers_reference as R  # noqa: E402

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def rand(*shape, seed=0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def draw_ids(n, vocab, how, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if how == "even":
        return torch.randint(vocab, (n,), generator=g, device="cuda")
    if how == "one":         # one token only
        return torch.full((n,), vocab // 2, dtype=torch.int64, device="cuda")
    if how == "few":         # a handful of frequent tokens and strays
        ids = torch.randint(min(3, vocab), (n,), generator=g, device="cuda")
        return torch.where(torch.rand(n, generator=g, device="cuda") < 0.05, torch.randint(vocab, (n,), generator=g, device="cuda"), ids)
    ids = torch.randint(-vocab // 2, 2 * vocab, (n,), generator=g, device="cuda")     # many that are no tokens
    ids[::7] = -(1 << 62)
    ids[3::11] = (1 << 40) + 1
    return ids


def check_forward(table, ids, scale, **k):
    out = B.adapt_embedding(table, ids, scale=scale, **k)
    want = R.embedding(table, ids.reshape(-1), scale).reshape(*ids.shape, table.shape[1])
    # one product in fp32 and the rounding to the type
    assert R.within(out, want, R.half_step(want, table.dtype) + R.U * want.abs() * 1.01)
    return out


def check_backward(dy, ids, vocab, scale, **k):
    grad = B.adapt_embedding_backward(dy, ids, vocab, scale=scale, **k)
    want, tol = R.embedding_gradient(dy.reshape(-1, dy.shape[-1]), ids.reshape(-1), vocab, scale)
    assert R.within(grad, want, R.half_step(want, grad.dtype) + 1.01 * tol)
    assert torch.equal(grad, B.adapt_embedding_backward(dy, ids, vocab, scale=scale, **k))
    return grad


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (5, 3, 7), (64, 1000, 64), (33, 50, 1001), (700, 40, 8), (3, 9, 20000), (2000, 300, 136)])
def test_forward(dtype, n, vocab, dim):
    table = rand(vocab, dim, dtype=dtype)
    check_forward(table, draw_ids(n, vocab, "even"), 1.0)
    check_forward(table, draw_ids(n, vocab, "wild"), -2.75)


@pytest.mark.parametrize("dtype", TYPES)
def test_forward_layouts(dtype):
    wide = rand(50, 100, dtype=dtype)
    ids = draw_ids(24, 50, "wild").reshape(2, 3, 4)
    for first, dim in ((0, 64), (1, 64), (8, 40), (3, 33)):
        table = wide[:, first:first + dim]
        check_forward(table, ids, 0.5)
        for at in (0, 1, 8):
            out = torch.full((24, 90), 7.0, dtype=dtype, device="cuda")
            got = check_forward(table, ids.reshape(-1), 0.5, out=out[:, at:at + dim])
            assert got.data_ptr() == out[:, at:].data_ptr()
            assert (out[:, :at] == 7).all() and (out[:, at + dim:] == 7).all()


def test_tokens_in_any_order():
    """A column of a batch of tokens, and a transposed batch."""
    table, batch = rand(30, 16), draw_ids(60, 30, "even").reshape(6, 10)
    for ids in (batch[:, 3], batch.t(), batch[::2]):
        assert torch.equal(B.adapt_embedding(table, ids), table[ids])
        dy = rand(*ids.shape, 16)
        assert torch.equal(B.adapt_embedding_backward(dy, ids, 30), B.adapt_embedding_backward(dy, ids.contiguous(), 30))


def test_values_pass_unchanged():
    table = torch.tensor([[math.inf, -math.inf, math.nan, 0.0, 1e-45]], device="cuda")
    out = B.adapt_embedding(table, torch.zeros(2, dtype=torch.int64, device="cuda"))
    assert torch.equal(out.nan_to_num(nan=5.0), table.nan_to_num(nan=5.0).expand(2, 5))


@pytest.mark.parametrize("dtype,grad", [(torch.float32, None), (torch.float16, None), (torch.bfloat16, None), (torch.float16, torch.float32),
                                        (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("how", ["even", "one", "few", "wild"])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 700, 8), (31, 5, 7), (64, 64, 64), (65, 1000, 33), (1000, 17, 136), (4099, 3001, 40),
                                         (20011, 70000, 8)])
def test_backward(dtype, grad, how, n, vocab, dim):
    check_backward(rand(n, dim, dtype=dtype), draw_ids(n, vocab, how), vocab, 1.5, dtype=grad)


@pytest.mark.parametrize("n,vocab,dim,how", [(300001, 513, 8, "few"), (262144, 300000, 4, "even"), (70001, 2, 16, "even"), (150000, 31, 24, "one"),
                                             (100000, (1 << 19) - 1, 1, "even"), (33000, 1 << 18, 3, "wild"), (1500, 700, 20000, "few")])
def test_backward_of_many(n, vocab, dim, how):
    check_backward(rand(n, dim, dtype=torch.bfloat16), draw_ids(n, vocab, how), vocab, 0.25, dtype=torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_backward_layouts(dtype):
    ids = draw_ids(301, 90, "few")
    wide = rand(301, 100, dtype=dtype)
    for first, dim in ((0, 64), (1, 64), (8, 40), (3, 33)):
        dy = wide[:, first:first + dim]
        want = check_backward(dy, ids, 90, 2.0)
        for at in (0, 1, 16):
            buf = torch.full((90, 120), 7.0, dtype=dtype, device="cuda")
            B.adapt_embedding_backward(dy, ids, 90, scale=2.0, dtable=buf[:, at:at + dim])
            assert torch.equal(buf[:, at:at + dim], want)
            assert (buf[:, :at] == 7).all() and (buf[:, at + dim:] == 7).all()
    check_backward(wide[:300].reshape(10, 30, 100), ids[:300].reshape(10, 30), 90, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_accumulation(dtype):
    ids, dy = draw_ids(500, 60, "wild"), rand(500, 48, dtype=dtype)
    for grad in {dtype, torch.float32}:
        start = rand(60, 48, seed=5, dtype=grad)
        got = B.adapt_embedding_backward(dy, ids, 60, scale=3.0, dtable=start.clone(), accumulate=True)
        want, tol = R.embedding_gradient(dy, ids, 60, 3.0)
        want = want + start.double()
        assert R.within(got, want, R.half_step(want, grad) + 1.01 * tol + R.U * want.abs())
        absent = torch.ones(60, dtype=torch.bool, device="cuda")
        absent[ids[(ids >= 0) & (ids < 60)]] = False
        assert torch.equal(got[absent], start[absent])


def test_rows_without_a_token_are_not_read():
    ids = draw_ids(2000, 50, "wild")
    dy = rand(2000, 24)
    want = B.adapt_embedding_backward(dy, ids, 50)
    dy[(ids < 0) | (ids >= 50)] = math.nan
    assert torch.equal(B.adapt_embedding_backward(dy, ids, 50), want)
    none = torch.full((77,), -1, dtype=torch.int64, device="cuda")
    assert (B.adapt_embedding_backward(dy[:77], none, 50) == 0).all()


def test_no_tokens():
    ids = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert B.adapt_embedding(rand(4, 8), ids).shape == (0, 8)
    assert (B.adapt_embedding_backward(rand(0, 8), ids, 9) == 0).all()
    start = rand(9, 8)
    assert torch.equal(B.adapt_embedding_backward(rand(0, 8), ids, 9, dtable=start.clone(), accumulate=True), start)


def test_gradient_against_differences():
    """<out(table + h d) - out(table - h d), dy> / 2h = <dtable, d>: the operator is linear, so the difference is exact
    but for roundings: u for each of the n dim products, and u / h where the outputs of size 2 are subtracted."""
    ids, h = draw_ids(90, 40, "few"), 2.0 ** -6
    table, dy, d = rand(40, 16), rand(90, 16, seed=1), rand(40, 16, seed=2)
    up, down = (B.adapt_embedding(table + s * h * d, ids, scale=2.0).double() for s in (1, -1))
    got = (B.adapt_embedding_backward(dy, ids, 40, scale=2.0).double() * d.double()).sum()
    want = ((up - down) * dy.double()).sum() / (2 * h)
    size = ((up.abs() + down.abs()) * dy.double().abs()).sum()
    assert abs(got - want) <= (4 / h + 100) * R.U * size


def test_streams_and_graphs():
    ids, dy, table = draw_ids(5000, 300, "few"), rand(5000, 64), rand(300, 64)
    want, out = B.adapt_embedding_backward(dy, ids, 300), B.adapt_embedding(table, ids)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.adapt_embedding_backward(dy, ids, 300, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graphs, grads, outs = [], [], []
    for _ in range(2):      # two graphs with scratch of their own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(B.adapt_embedding(table, ids))
            grads.append(B.adapt_embedding_backward(dy, ids, 300))
        graphs.append(g)
    new = draw_ids(5000, 300, "even", seed=9)
    ids.copy_(new)
    graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    want, out = B.adapt_embedding_backward(dy, ids, 300), B.adapt_embedding(table, ids)
    for a, b in zip(grads, outs):
        assert torch.equal(a, want) and torch.equal(b, out)


def test_refusals():
    table, ids, dy = rand(10, 8), draw_ids(4, 10, "even"), rand(4, 8)
    for call in (lambda: B.adapt_embedding(table.double(), ids), lambda: B.adapt_embedding(table, ids.int()), lambda: B.adapt_embedding(table, ids.cpu()),
                 lambda: B.adapt_embedding(table.t(), ids), lambda: B.adapt_embedding(table[0], ids), lambda: B.adapt_embedding(table, ids, out=dy.half()),
                 lambda: B.adapt_embedding(table, ids, out=dy[:3]), lambda: B.adapt_embedding_backward(dy[:3], ids, 10),
                 lambda: B.adapt_embedding_backward(dy, ids, 10, accumulate=True), lambda: B.adapt_embedding_backward(dy, ids, 10, dtable=table[:9]),
                 lambda: B.adapt_embedding_backward(dy, ids, 10, dtable=table.half()), lambda: B.adapt_embedding_backward(dy, ids, 10, dtype=torch.float64),
                 lambda: B.adapt_embedding_backward(dy, ids, -1), lambda: B.adapt_embedding_backward(dy, ids.float(), 10)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: B.adapt_embedding_backward(dy, ids, 0), lambda: B.adapt_embedding(table, ids, scale=math.inf),
                 lambda: B.adapt_embedding_backward(dy, ids, 10, dtype=torch.float16)):
        with pytest.raises(B.AdaptError) as e:
            call()
        assert e.value.status == B.ERR_INVALID_ARG
