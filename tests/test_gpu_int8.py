"""Rows to 8-bit codes and the product of codes, against their definitions in 64 bits."""
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


def codes(*shape, seed=0, least=-128):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(least, 128, shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int8)


def positive(n, seed=0):
    return rand(n, seed=seed).abs() * 0.01 + 1e-3


def check(x, w, w_scales, x_scales=None, bias=None, **k):
    y = B.adapt_int8_linear(x, w, w_scales, x_scales=x_scales, bias=bias, **k)
    c, s = (x, x_scales) if x.dtype == torch.int8 else R.int8_rows(x)
    want, tol = R.int8_linear(c, s, w, w_scales, bias)
    assert R.within(y, want, tol + R.half_step(want, y.dtype) * 1.01)
    return y


def same_codes(r, x):
    want, scales = R.int8_rows(x)
    assert torch.equal(r.codes.double(), want)
    assert torch.equal(r.scales.nan_to_num(nan=-1.0), scales.nan_to_num(nan=-1.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 64), (2, 1000), (700, 33), (9, 4096), (2, 16384), (2, 40001)])
def test_rows(dtype, rows, cols):
    x = rand(rows, cols, dtype=dtype)
    x[:, ::13] *= 9
    same_codes(B.adapt_int8_rows(x), x)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_next_to_ties(dtype):
    """Values on and next to the middle between two codes, for many largest values."""
    rows = []
    for i in range(64):
        m = 1.0 + i / 64
        half = (torch.arange(-126, 127, dtype=torch.float64) + 0.5) * m / 127
        rows.append(torch.cat([half, torch.tensor([m], dtype=torch.float64)]))
    x = torch.stack(rows).to(dtype).cuda()
    if dtype == torch.float32:
        x = torch.cat([x, torch.nextafter(x, torch.full_like(x, 9.0)), torch.nextafter(x, torch.full_like(x, -9.0))])
    same_codes(B.adapt_int8_rows(x), x)


def test_rows_of_extreme_values():
    x = rand(12, 300)
    x[0] = 0
    x[1] *= 1e-38
    x[2] *= 1e-44
    x[3, 5] = math.nan
    x[4, 299] = math.inf
    x[5, 0] = -math.inf
    x[6] = 3e38
    x[7] *= 1e-30
    x[8] = -0.0
    r = B.adapt_int8_rows(x)
    same_codes(r, x)
    assert r.scales[3:6].isnan().all() and (r.codes[3:6] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_layouts(dtype):
    wide = rand(20, 200, dtype=dtype)
    for first, cols in ((0, 128), (1, 128), (8, 100), (3, 97)):
        x = wide[:, first:first + cols]
        for at in (0, 1, 16):
            out = torch.full((20, 220), 99, dtype=torch.int8, device="cuda")
            r = B.adapt_int8_rows(x, codes=out[:, at:at + cols])
            same_codes(r, x)
            assert (out[:, :at] == 99).all() and (out[:, at + cols:] == 99).all()
    x = wide[:1].expand(5, 200)     # one row for all
    same_codes(B.adapt_int8_rows(x), x)


SIZES = [(1, 1, 1), (1, 64, 128), (1, 1000, 4096), (2, 33, 100), (3, 128, 16), (7, 300, 2048), (16, 256, 256), (17, 500, 1001), (64, 1024, 512),
         (65, 130, 96), (100, 100, 1000), (128, 256, 128), (129, 257, 144), (200, 1531, 320), (333, 512, 4096), (513, 640, 80), (1000, 384, 2050)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,k", SIZES)
def test_product(dtype, rows, n, k):
    w = codes(n, k)
    check(codes(rows, k, seed=1), w, positive(n), positive(rows, 2), dtype=dtype)
    check(codes(rows, k, seed=3), w, positive(1), positive(1, 2), bias=rand(n), dtype=dtype)
    for x_type in TYPES:
        check(rand(rows, k, seed=4, dtype=x_type), w, positive(n), dtype=dtype)


@pytest.mark.parametrize("rows", [1, 5, 40, 300])
def test_extreme_codes_are_exact(rows):
    """The largest sum that a product can have, and sums of one sign."""
    k = 131071
    one = torch.ones(1, device="cuda")
    low = torch.full((1, k), -128, dtype=torch.int8, device="cuda")
    x, w = low.expand(rows, k), torch.cat([low, -low - 1, low])
    y = B.adapt_int8_linear(x, w, one, x_scales=one)
    for j, sum_ in enumerate((128 * 128 * k, -127 * 128 * k, 128 * 128 * k)):
        assert (y[:, j] == torch.tensor(float(sum_), dtype=torch.float32, device="cuda")).all()


@pytest.mark.parametrize("rows", [1, 9, 70, 300])
def test_layouts(rows):
    """Slices with any alignment of x, the weights and y."""
    n, k = 200, 272
    xw, ww = codes(rows, k + 40, seed=1), codes(n, k + 40)
    fw = rand(rows, k + 40, seed=2, dtype=torch.bfloat16)
    for ax, aw, ay in ((0, 0, 0), (1, 0, 0), (0, 1, 0), (16, 16, 8), (3, 5, 1), (8, 4, 3)):
        out = torch.full((rows, n + 30), 5.0, dtype=torch.bfloat16, device="cuda")
        y = out[:, ay:ay + n]
        check(xw[:, ax:ax + k], ww[:, aw:aw + k], positive(n), positive(rows, 3), out=y)
        assert (out[:, :ay] == 5).all() and (out[:, ay + n:] == 5).all()
        check(fw[:, ax:ax + k], ww[:, aw:aw + k], positive(n), out=y)
        assert (out[:, :ay] == 5).all() and (out[:, ay + n:] == 5).all()
    check(xw[:1, :k].expand(rows, k), ww[:1, :k].expand(n, k), positive(n), positive(rows))


def test_rows_with_nan_stay_alone():
    for rows in (3, 200):
        x, w = rand(rows, 256), codes(128, 256)
        x[1, 7] = math.nan
        y = check(x, w, positive(128))
        assert y[1].isnan().all() and not y[0].isnan().any()


def test_empty():
    one = torch.ones(1, device="cuda")
    assert B.adapt_int8_linear(codes(0, 8), codes(5, 8), one, x_scales=one).shape == (0, 5)
    assert B.adapt_int8_linear(codes(3, 8), codes(0, 8), one, x_scales=one).shape == (3, 0)
    b = rand(5)
    assert torch.equal(B.adapt_int8_linear(codes(3, 0), codes(5, 0), one, x_scales=one, bias=b), b.expand(3, 5))
    assert torch.equal(B.adapt_int8_linear(rand(3, 0), codes(5, 0), one, bias=b), b.expand(3, 5))
    assert B.adapt_int8_rows(rand(0, 8)).codes.shape == (0, 8)


@pytest.mark.parametrize("rows", [1, 100])
def test_fixed_point_weights(rows):
    """Codes of adapt_quantize at <8, FL> with the scale 2^-FL: the product of the dequantized weights."""
    w = rand(96, 160) * 0.3
    q = B.adapt_quantize_ex(w.reshape(-1), 8, 7, code_bits=8).reshape(96, 160)
    x = rand(rows, 160, seed=1)
    y = check(x, q, torch.full((1,), 2.0 ** -7, device="cuda"))
    c, s = R.int8_rows(x)
    exact = (c * s.double()[:, None]) @ (q.double() * 2.0 ** -7).t()
    assert R.within(y, exact, 4 * R.U * exact.abs() + 2.0 ** -140)


def test_streams_and_graphs():
    for rows in (2, 40, 300):
        x, w, s = rand(rows, 512, dtype=torch.bfloat16), codes(640, 512), positive(640)
        want = B.adapt_int8_linear(x, w, s)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = B.adapt_int8_linear(x, w, s, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = B.adapt_int8_linear(x, w, s)
            graphs.append((graph, out))
        x.mul_(-0.5)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = B.adapt_int8_linear(x, w, s)
        assert all(torch.equal(out, want) for _, out in graphs)


def test_refusals():
    x, w, one = rand(4, 32), codes(6, 32), torch.ones(1, device="cuda")
    c = codes(4, 32)
    for call in (lambda: B.adapt_int8_linear(x.double(), w, one), lambda: B.adapt_int8_linear(x, w.float(), one), lambda: B.adapt_int8_linear(x[:, :31], w, one),
                 lambda: B.adapt_int8_linear(x, w, one.half()), lambda: B.adapt_int8_linear(x, w, one.expand(5)), lambda: B.adapt_int8_linear(x, w, one, x_scales=one),
                 lambda: B.adapt_int8_linear(c, w, one), lambda: B.adapt_int8_linear(c, w, one, x_scales=one.cpu()), lambda: B.adapt_int8_linear(x, w.t(), one),
                 lambda: B.adapt_int8_linear(x, w, one, bias=rand(5)), lambda: B.adapt_int8_linear(x, w, one, dtype=torch.int8),
                 lambda: B.adapt_int8_linear(x, w, one, out=rand(4, 5)), lambda: B.adapt_int8_linear(x, w.cpu(), one), lambda: B.adapt_int8_rows(c),
                 lambda: B.adapt_int8_rows(x, codes=c[:3]), lambda: B.adapt_int8_rows(x.t()), lambda: B.adapt_int8_rows(x, scales=one)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(B.AdaptError) as e:
        B.adapt_int8_linear(codes(2, 1).new_zeros(2, B.INT8_MAX_K + 1), codes(1, 1).new_zeros(2, B.INT8_MAX_K + 1), one, x_scales=one)
    assert e.value.status == B.ERR_INVALID_ARG
