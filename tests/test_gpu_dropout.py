"""Dropout against the 64-bit reference: the mask bit for bit, the values to a derived bound.

Bound: y is x times a rounded scale (two roundings of 2^-24), a sum with the residual (one more) and
one rounding to the element type: |error| <= (u + 2^-21) (|x s| + |r|) + the type's smallest number,
u = 2^-24, 2^-11, 2^-8 for fp32, fp16, bf16."""
import numpy as np
import pytest

from tests import training_reference as R

pytestmark = pytest.mark.gpu

UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -133}


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2107_13490_b200 import binding
    binding.lib()
    return binding


def check(y, x, r, p, keep, dtype):
    y, x = y.double().cpu().numpy().ravel(), x.double().cpu().numpy().ravel()
    want = np.where(keep, x / (1 - p) if p < 1 else 0.0, 0.0)
    size = np.abs(want)
    if r is not None:
        r = r.double().cpu().numpy().ravel()
        want, size = want + r, size + np.abs(r)
    tol = (UNIT[dtype] + 2.0 ** -21) * size + TINY[dtype]
    assert (np.abs(y - want) <= tol).all()
    if r is None:
        assert (y[~keep] == 0).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 255, 1025, 4099, 20011])
def test_flat(B, dtype, n):
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, generator=g, device="cuda").to(getattr(torch, dtype))
    r = torch.randn(n, generator=g, device="cuda").to(x.dtype)
    for p, seed, layer, base in ((0.1, 3, 0, 0), (0.5, 2 ** 63 + 11, 4, 1), (0.9, 5, -2, 2 ** 40 + 3)):
        keep = R.dropout_keep(n, p, seed, layer, base)
        check(B.adapt_dropout(x, p, seed, layer, base), x, None, p, keep, dtype)
        check(B.adapt_dropout(x, p, seed, layer, base, residual=r), x, r, p, keep, dtype)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (5, 1, 3), (3, 10, 0), (7, 33, 7), (13, 129, 7), (4, 1000, 24),
                                           (33, 64, 64), (64, 65, 0), (2, 4097, 1)])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_rows_strides_and_offsets(B, dtype, rows, cols, pad, shift):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows * cols)
    dt = getattr(torch, dtype)

    def matrix(pad, shift):
        ld = cols + pad
        buf = torch.randn(rows * ld + 8, generator=g, device="cuda").to(dt)
        return buf, torch.as_strided(buf, (rows, cols), (ld, 1), shift)

    keep = R.dropout_keep(rows * cols, 0.3, 77, 2)
    (_, x), (_, r) = matrix(pad, shift), matrix(pad, shift)
    for out_pad, out_shift in ((pad, shift), (pad + 1, 0), (0, shift)):   # the last two: other alignments
        buf, y = matrix(out_pad, out_shift)
        before = buf.clone()
        B.adapt_dropout(x, 0.3, 77, 2, residual=r, out=y)
        check(y, x, r, 0.3, keep, dtype)
        B.adapt_dropout(x, 0.3, 77, 2, out=y)
        check(y, x, None, 0.3, keep, dtype)
        y.copy_(torch.as_strided(before, y.shape, y.stride(), out_shift))   # nothing beside y was written
        assert torch.equal(buf.view(torch.uint8), before.view(torch.uint8))


def test_dropped_elements_count_as_zero_whatever_they_hold(B):
    import torch
    n = 4096
    keep = torch.from_numpy(R.dropout_keep(n, 0.5, 1, 0)).cuda()
    for dt in (torch.float32, torch.float16, torch.bfloat16):
        x = torch.where(keep, torch.ones(n, device="cuda"), torch.full((n,), float("nan"), device="cuda")).to(dt)
        x[::3] = torch.where(keep[::3], x[::3], torch.full_like(x[::3], float("-inf")))
        y = B.adapt_dropout(x, 0.5, 1, 0)
        assert torch.equal(y, torch.where(keep, 2.0, 0.0).to(dt))
        r = torch.full_like(x, 0.25)
        assert torch.equal(B.adapt_dropout(x, 0.5, 1, 0, residual=r), torch.where(keep, 2.25, 0.25).to(dt))
        bad = B.adapt_dropout(torch.full((n,), float("nan"), device="cuda", dtype=dt), 1.0, 1, 0, residual=r)
        assert torch.equal(bad, r)


def test_probabilities_of_zero_and_one(B):
    import torch
    x = torch.randn(1000, device="cuda")
    assert torch.equal(B.adapt_dropout(x, 0.0, 9), x)
    assert torch.equal(B.adapt_dropout(x, 1.0, 9), torch.zeros_like(x))
    assert (B.adapt_dropout(x, 1e-30, 9) == x).all()


def test_in_place_stream_and_views_give_the_same_mask(B):
    import torch
    x = torch.randn(64, 96, device="cuda").bfloat16()
    r = torch.randn_like(x)
    want = B.adapt_dropout(x, 0.2, 8, 1, residual=r)
    assert torch.equal(B.adapt_dropout(x.reshape(8, 8, 96), 0.2, 8, 1, residual=r.reshape(8, 8, 96)).reshape(64, 96), want)
    wide = torch.zeros(64, 128, device="cuda", dtype=x.dtype)
    wide[:, :96] = x
    assert torch.equal(B.adapt_dropout(wide[:, :96], 0.2, 8, 1, residual=r), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = B.adapt_dropout(x, 0.2, 8, 1, residual=r, stream=s)
    s.synchronize()
    assert torch.equal(other, want)
    # halves with an index base draw the whole's mask
    flat, fr = x.reshape(-1), r.reshape(-1)
    half = torch.cat([B.adapt_dropout(flat[:3001].clone(), 0.2, 8, 1, 0, fr[:3001].clone()),
                      B.adapt_dropout(flat[3001:].clone(), 0.2, 8, 1, 3001, fr[3001:].clone())])
    assert torch.equal(half, want.reshape(-1))
    a, b = x.clone(), r.clone()
    assert torch.equal(B.adapt_dropout(a, 0.2, 8, 1, residual=r, out=a), want)
    assert torch.equal(B.adapt_dropout(x, 0.2, 8, 1, residual=b, out=b), want)


def test_gradient_is_the_same_call(B):
    import torch
    # y is linear in x: the difference quotient of sum(w y) along v is sum(v dropout(w)) up to rounding
    x, v, w = (torch.randn(5000, device="cuda") for _ in range(3))
    f = lambda t: (B.adapt_dropout(t, 0.25, 3, 3).double() * w.double()).sum()  # noqa: E731
    eps = 0.5
    diff = (f(x + eps * v) - f(x - eps * v)) / (2 * eps)
    grad = (B.adapt_dropout(w, 0.25, 3, 3).double() * v.double()).sum()
    size = (w.abs() * (x.abs() + v.abs())).double().sum() / 0.75
    assert abs(diff - grad) <= 2.0 ** -21 * size / eps


def test_large_tensor_samples(B):
    import torch
    n = (1 << 26) + 5
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    y = B.adapt_dropout(x, 0.5, 21, 1)
    for start in (0, 12345678, n - 64):
        assert np.array_equal(y[start:start + 64].float().cpu().numpy() != 0, R.dropout_keep(64, 0.5, 21, 1, start))
    assert abs(float((y != 0).double().mean()) - 0.5) < 5 * 0.5 / n ** 0.5


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("cols", [3, 8, 37, 256, 1003])
def test_every_pair_of_alignments(B, dtype, cols):
    import torch
    dt = getattr(torch, dtype)
    lane = 16 // torch.empty(0, dtype=dt).element_size()
    rows = 5
    keep = R.dropout_keep(rows * cols, 0.4, 12, 3)
    g = torch.Generator(device="cuda").manual_seed(cols)

    def matrix(shift, pad):
        # the matrix ends where its buffer ends, so that a read beyond it would leave the buffer
        buf = torch.randn(shift + (rows - 1) * (cols + pad) + cols, generator=g, device="cuda").to(dt)
        return buf, torch.as_strided(buf, (rows, cols), (cols + pad, 1), shift)

    for shift in range(lane):
        _, x = matrix(shift, 3)
        _, r = matrix((3 * shift + 1) % lane, 5)
        for pad in (0, 2):
            buf, y = matrix((shift * 5 + 2) % lane, pad)
            before = buf.clone()
            check(B.adapt_dropout(x, 0.4, 12, 3, residual=r, out=y), x, r, 0.4, keep, dtype)
            y.copy_(torch.as_strided(before, y.shape, y.stride(), y.storage_offset()))
            assert torch.equal(buf.view(torch.uint8), before.view(torch.uint8))
        for same in (x, r):   # in place, the other operand at another alignment
            want = B.adapt_dropout(x, 0.4, 12, 3, residual=r)
            held = same.clone()
            assert torch.equal(B.adapt_dropout(x, 0.4, 12, 3, residual=r, out=same), want)
            same.copy_(held)
    line, other = matrix(1, 0)[1].reshape(-1), matrix(2, 0)[1].reshape(-1)   # one long row
    check(B.adapt_dropout(line, 0.4, 12, 3, residual=other), line, other, 0.4, keep, dtype)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("cols", [1, 2, 5, 10, 15, 16, 17])
def test_short_rows_of_other_alignments(B, dtype, cols):
    import torch
    dt, rows = getattr(torch, dtype), 700       # more than a CTA's pairs
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(rows, cols + 3, generator=g, device="cuda").to(dt)[:, 1:1 + cols]
    r = torch.randn(rows, cols + 2, generator=g, device="cuda").to(dt)[:, 2:]
    for base in (0, 7):
        keep = R.dropout_keep(rows * cols, 0.3, 5, 6, base)
        out = torch.full((rows, cols + 5), 7.0, device="cuda", dtype=dt)
        y = out[:, 3:3 + cols]
        check(B.adapt_dropout(x, 0.3, 5, 6, base, out=y), x, None, 0.3, keep, dtype)
        check(B.adapt_dropout(x, 0.3, 5, 6, base, residual=r, out=y), x, r, 0.3, keep, dtype)
        assert (out[:, :3] == 7).all() and (out[:, 3 + cols:] == 7).all()
    want = B.adapt_dropout(x, 0.3, 5, 6, 7, residual=r)
    for same in (x, r):
        held = same.clone()
        assert torch.equal(B.adapt_dropout(x, 0.3, 5, 6, 7, residual=r, out=same), want)
        same.copy_(held)
    assert torch.equal(B.adapt_dropout(x, 1.0, 5, 6, residual=r, out=y), r)
    assert torch.equal(B.adapt_dropout(x, 0.0, 5, 6, out=y), x)
    x[::2] = float("nan")
    y = B.adapt_dropout(x, 0.3, 5, 6, out=y).float().cpu().numpy().ravel()
    assert np.array_equal(np.isnan(y), R.dropout_keep(rows * cols, 0.3, 5, 6) & np.repeat(np.arange(rows) % 2 == 0, cols))
