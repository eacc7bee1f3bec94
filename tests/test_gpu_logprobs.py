"""Token log probabilities against the 64-bit reference.

Bounds (fp32 arithmetic).  An exponent z - m carries an error of 2^-22 Z, Z the largest |z| that
matters (p > 1e-30); the exponential 2^-22; a sum of V terms in at least 32 chains (V / 32 + 32) 2^-24.
So ln s is off by at most t = 2^-21 (2 + Z) + (V / 32 + 32) 2^-24, lse by t + 2^-23 |lse|, a log probability by
twice that, the entropy by 2 t (2 + ln V + spread), spread = sum p |ln p|.  A gradient's p is off by
2 t relatively, and is rounded once."""
import math

import numpy as np
import pytest

from tests import training_reference as R

pytestmark = pytest.mark.gpu

UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -126, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -126}   # bound for subnormal results
DTYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2107_13490_b200 import binding
    binding.lib()
    return binding


def close(got, want, tol):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf])
    fine = np.isfinite(want)
    err = np.abs(got[fine] - want[fine])
    assert (err <= np.broadcast_to(tol, want.shape)[fine]).all(), float((err / np.broadcast_to(tol, want.shape)[fine]).max())


def slack(x, scale, lse):
    z = R.scaled(x, scale)
    with np.errstate(invalid="ignore"):
        big = np.where(z - lse[:, None] > -70, np.abs(z), 0.0)
    big = np.nan_to_num(big, nan=0.0, posinf=0.0).max(1)
    return 2.0 ** -21 * (2 + big) + (x.shape[1] / 32 + 32) * 2.0 ** -24, big


def compare(B, x, t, scale=1.0, k=0, weights=True, out_pad=0):
    """x: torch matrix; t: list of targets or None."""
    import torch
    dtype = str(x.dtype).split(".")[1]
    xd = x.double().cpu().numpy()
    rows, vocab = xd.shape
    td = None if t is None else torch.tensor(t, dtype=torch.int64, device="cuda")
    want = R.logprobs(xd, t, scale, k)
    tol, big = slack(xd, scale, want["lse"])
    lse_tol = tol + 2.0 ** -23 * np.nan_to_num(np.abs(want["lse"]), nan=0, posinf=0, neginf=0)
    spread = np.zeros(rows)
    ent_tol = 2 * tol * (2 + 2 * math.log(max(vocab, 2)))
    rng = np.random.default_rng(rows * vocab)
    dlp, dh = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    gl, gh = torch.from_numpy(dlp).cuda(), torch.from_numpy(dh).cuda()

    def stats(r):
        close(r.lse, want["lse"], lse_tol)
        if t is not None:
            close(r.logprob, want["logprob"], 2 * lse_tol + 2.0 ** -22 * big)
        close(r.entropy, want["entropy"], ent_tol)
        if k:
            assert np.array_equal(r.top_ids.cpu().numpy(), want["top_ids"])
            close(r.top_logprobs, want["top_logprobs"], (2 * lse_tol + 2.0 ** -22 * big)[:, None] +
                  2.0 ** -22 * np.where(np.isfinite(want["top_logprobs"]), np.abs(want["top_logprobs"]), 0))

    r = B.adapt_token_logprobs(x, td, scale=scale, n_top=k)
    stats(r)
    if not weights:
        return r

    def gradient(g, dl, dh):
        ref = R.logprobs_gradient(xd, t, scale, want["lse"], want["entropy"], dl, dh)
        with np.errstate(invalid="ignore", over="ignore"):
            lse = np.where(np.isfinite(want["lse"]), want["lse"], 0)[:, None]
            logp = np.where(np.isfinite(R.scaled(xd, scale)), xd * scale - lse, -1e4)
            p = np.exp(np.minimum(logp, 0))
        a = 0 if dl is None else np.abs(dl)[:, None]
        b = 0 if dh is None else np.abs(dh)[:, None]
        h = np.where(np.isfinite(want["entropy"]), want["entropy"], 0)[:, None]
        rel = (2 * lse_tol + 2.0 ** -22 * (big + 2))[:, None]
        tol = scale * p * (a * rel + b * ((np.abs(logp) + h) * rel + rel + ent_tol[:, None]))
        tol = tol + scale * (a + 0) * 2.0 ** -22 + UNIT[dtype] * np.nan_to_num(np.abs(ref)) + TINY[dtype]
        close(g, ref, tol)

    ld = vocab + out_pad
    combos = [(None, gh)] if t is None else [(gl, None), (None, gh), (gl, gh)]
    for a, b in combos:
        na, nb = None if a is None else dlp, None if b is None else dh
        out = torch.empty(rows, ld, dtype=x.dtype, device="cuda")[:, :vocab]
        both = B.adapt_token_logprobs(x, td, scale=scale, n_top=k, d_logprob=a, d_entropy=b, dlogits=out)
        stats(both)
        gradient(both.dlogits, na, nb)
        gradient(B.adapt_token_logprobs_backward(x, td, r.lse, a, r.entropy, b, scale=scale), na, nb)
    return r


def logits(rows, vocab, dtype, seed, spread=3.0, pad=0, shift=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = vocab + pad
    buf = (torch.randn(rows * ld + 8, generator=g, device="cuda") * spread).to(getattr(torch, dtype))
    return torch.as_strided(buf, (rows, vocab), (ld, 1), shift)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (128, 10), (5, 100), (33, 257), (7, 1000), (2, 2049), (3, 4097),
                                        (2, 9001), (1, 20000), (300, 1031)])
def test_sizes(B, dtype, rows, vocab):
    x = logits(rows, vocab, dtype, rows + vocab)
    rng = np.random.default_rng(vocab)
    t = rng.integers(0, vocab, rows)
    t[::5] = -1
    t[-1] = vocab - 1
    compare(B, x, t.tolist(), k=min(vocab, 5), weights=rows * vocab < 50000)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift,out_pad", [(1, 0, 1), (7, 3, 0), (0, 1, 0), (8, 0, 8), (3, 5, 2)])
def test_strides_and_offsets(B, dtype, pad, shift, out_pad):
    for vocab in (9, 515, 2500):
        x = logits(4, vocab, dtype, vocab, pad=pad, shift=shift)
        compare(B, x, [0, vocab - 1, -1, vocab // 2], scale=0.7, k=4, out_pad=out_pad)


@pytest.mark.parametrize("k", [1, 2, 8, 20, 32])
@pytest.mark.parametrize("vocab", [32, 300, 5000])
def test_alternatives_with_ties(B, k, vocab):
    import torch
    for seed, levels in ((0, 3), (1, 40), (2, 1)):   # few distinct values: ties go to the lowest index
        rng = np.random.default_rng(seed)
        x = torch.from_numpy(rng.integers(0, levels, (5, vocab)).astype(np.float32)).cuda()
        x[1] = -x[1]          # holds -0.0 beside 0.0
        x[1, ::2] *= -1.0
        compare(B, x, [0] * 5, k=k, weights=False)
        compare(B, x.bfloat16(), None, k=k, weights=False)


@pytest.mark.parametrize("vocab", [64, 6000])
def test_alternatives_of_sorted_and_clustered_rows(B, vocab):
    import torch
    up = torch.linspace(-3, 9, vocab, device="cuda")
    block = torch.zeros(vocab, device="cuda")
    n = min(40, vocab // 2)
    block[vocab // 2:vocab // 2 + n] = torch.arange(n, device="cuda") * 0.01 + 5   # neighbours hold the largest
    stride = torch.zeros(vocab, device="cuda")
    stride[3::64] = torch.arange(stride[3::64].numel(), device="cuda") * 0.01 + 5    # every 64th
    x = torch.stack([up, up.flip(0), block, stride])
    compare(B, x, [0, 1, 2, 3], k=32, weights=False)
    compare(B, x.half(), [0, 1, 2, 3], k=32, weights=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [40, 3000])
def test_barred_logits_and_empty_rows(B, dtype, vocab):
    import torch
    x = logits(8, vocab, dtype, 5)
    low = torch.finfo(x.dtype).min
    x[0, 1:] = -math.inf                      # one token left
    x[1] = -math.inf                          # nothing left
    x[2, ::2] = -math.inf
    x[3, ::2] = low
    x[4] = low                                # all the same: uniform
    x[5, :vocab // 2] = low
    x[5, vocab // 2:] = -math.inf
    x[6] = -math.inf
    t = [0, 3, 1, 1, 2, 0, -1, 4]
    compare(B, x, t, k=6)
    compare(B, x, t, scale=2.5 if dtype != "float32" else 0.5, k=3)
    compare(B, x, None, k=3)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_magnitudes(B, dtype):
    import torch
    top = float(torch.finfo(getattr(torch, dtype)).max)
    x = logits(4, 700, dtype, 3)
    x[0] *= 60 if dtype == "float16" else 1e4
    x[1, 5] = top
    x[2] = top
    compare(B, x, [1, 5, 2, 3], k=3, weights=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [50, 2600])
def test_nan_and_inf(B, dtype, vocab):
    x = logits(5, vocab, dtype, 8)
    x[0, 7] = math.nan
    x[1, 9] = math.inf
    x[2, 3] = math.inf
    x[2, 11] = math.nan
    x[3, 20] = -math.nan
    compare(B, x, [7, 0, 3, 1, 2], k=4, weights=False)
    import torch
    t = torch.tensor([7, 0, 3, 1, 2], device="cuda")
    d = torch.ones(5, device="cuda")
    r = B.adapt_token_logprobs(x, t, d_logprob=d, d_entropy=d)
    assert r.dlogits[:4].isnan().all() and r.dlogits[4].isfinite().all()


@pytest.mark.parametrize("rows,vocab", [(1100, 1500), (1100, 7777), (40, 7777)])
def test_special_rows_among_many(B, rows, vocab):
    import torch
    x = logits(rows, vocab, "bfloat16", 6)
    x[3] = -math.inf
    x[5, 17] = math.nan
    x[6, :] = torch.finfo(x.dtype).min
    x[7, 5:] = -math.inf
    x[9] = 1.0
    x[11, ::2] = -math.inf
    t = torch.arange(rows, device="cuda") % 5
    t[13] = -1
    t[14] = vocab
    d, e = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    r = B.adapt_token_logprobs(x, t, n_top=9, d_logprob=d, d_entropy=e)
    s = B.adapt_token_logprobs_backward(x, t, r.lse, d, r.entropy, e)
    for i in (2, 3, 5, 6, 7, 9, 11, 13, 14, 15):   # a row alone takes another form of the kernel
        one = B.adapt_token_logprobs(x[i:i + 1], t[i:i + 1], n_top=9, d_logprob=d[i:i + 1], d_entropy=e[i:i + 1])
        assert torch.equal(r.top_ids[i], one.top_ids[0])
        pairs = [(r.lse, one.lse), (r.entropy, one.entropy), (r.logprob, one.logprob),
                 (r.top_logprobs, one.top_logprobs), (r.dlogits.float(), one.dlogits.float())]
        if i != 6:   # (an fp32 lse of -3.4e38 does not hold ln vocab, so the gradient from it cannot either)
            pairs.append((s.float(), one.dlogits.float()))
        for a, b in pairs:
            # the same sums in another order: 2^-17 of values up to 20, and two roundings of a gradient
            assert torch.allclose(a[i], b[0], rtol=2.0 ** -7, atol=20 * 2.0 ** -17, equal_nan=True), i


def test_targets_outside_the_vocabulary(B):
    import torch
    x = logits(4, 300, "float32", 1)
    t = torch.tensor([-1, 300, -9 * 10 ** 17, 299], device="cuda")
    d = torch.ones(4, device="cuda")
    x[0, 3] = math.nan     # a row without a target is not read
    r = B.adapt_token_logprobs(x, t, n_top=2, d_logprob=d, d_entropy=d)
    assert r.logprob.isnan().tolist() == [False, True, False, False]
    assert r.lse.isfinite().all() and r.top_ids[0].tolist() == [-1, -1]
    assert (r.dlogits[0] == 0).all() and r.dlogits[1].isnan().all() and (r.dlogits[2] == 0).all()
    g = B.adapt_token_logprobs_backward(x, t, r.lse, d, r.entropy, d)
    assert torch.equal(g.isnan(), r.dlogits.isnan()) and (g[0] == 0).all()
    r = B.adapt_token_logprobs(x[1:], t[1:], d_entropy=d[1:])   # without a weight on the log probability
    assert r.dlogits.isfinite().all()


@pytest.mark.parametrize("vocab", [200, 5001])
def test_in_place_and_other_stream(B, vocab):
    import torch
    x = logits(37, vocab, "bfloat16", 4)
    t = torch.arange(37, device="cuda")
    d = torch.randn(37, device="cuda")
    want = B.adapt_token_logprobs(x, t, n_top=3, d_logprob=d, d_entropy=d)
    y = x.clone()
    got = B.adapt_token_logprobs(y, t, n_top=3, d_logprob=d, d_entropy=d, dlogits=y)
    assert torch.equal(y, want.dlogits) and torch.equal(got.lse, want.lse) and torch.equal(got.top_ids, want.top_ids)
    y = x.clone()
    back = B.adapt_token_logprobs_backward(x, t, want.lse, d, want.entropy, d)
    assert torch.equal(B.adapt_token_logprobs_backward(y, t, want.lse, d, want.entropy, d, out=y), back)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = B.adapt_token_logprobs(x, t, n_top=3, d_logprob=d, d_entropy=d, stream=s)
    s.synchronize()
    assert torch.equal(other.dlogits, want.dlogits) and torch.equal(other.entropy, want.entropy)


def test_gradient_against_differences(B):
    import torch
    rows, vocab, eps = 6, 800, 2.0 ** -6
    g = torch.Generator(device="cuda").manual_seed(0)
    x, v = (torch.randn(rows, vocab, generator=g, device="cuda") for _ in range(2))
    t = torch.tensor([0, 5, -1, 799, 3, 77], device="cuda")
    dl, dh = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))

    def value(x):
        r = B.adapt_token_logprobs(x, t)
        return (r.logprob.double() * dl.double() + r.entropy.double() * dh.double()).sum()

    d = (value(x + eps * v) - value(x - eps * v)) / (2 * eps)
    r = B.adapt_token_logprobs(x, t, d_logprob=dl, d_entropy=dh)
    # rounding: 12 values off by about 2^-21 of 10 each; truncation: eps^2 / 6 times third derivatives of order 10
    tol = 12 * 10 * 2.0 ** -21 / (2 * eps) * 2 + eps ** 2 / 6 * 10 * rows
    assert abs(d - (r.dlogits.double() * v.double()).sum()) <= tol


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 131072, "bfloat16"), (3, 250001, "float16"), (64, 32000, "float32"),
                                              (700, 40000, "bfloat16"), (1030, 8191, "float16"), (2100, 1025, "bfloat16"),
                                              (1024, 5000, "float32")])
def test_large_rows_against_64_bits_on_the_device(B, rows, vocab, dtype):
    import torch
    x = logits(rows, vocab, dtype, 2)
    t = torch.randint(vocab, (rows,), device="cuda")
    d = torch.randn(rows, device="cuda")
    r = B.adapt_token_logprobs(x, t, n_top=20, d_logprob=d, d_entropy=d)
    again = B.adapt_token_logprobs(x, t, n_top=20, d_logprob=d, d_entropy=d)
    assert torch.equal(r.lse, again.lse) and torch.equal(r.dlogits, again.dlogits)
    xd = x.double()
    logp = torch.log_softmax(xd, 1)
    p = logp.exp()
    h = -(p * logp).sum(1)
    tol = 2.0 ** -21 * (2 + float(xd.abs().max())) + (vocab / 32 + 32) * 2.0 ** -24
    assert ((r.logprob - logp.gather(1, t[:, None])[:, 0]).abs() <= 3 * tol).all()
    assert ((r.entropy - h).abs() <= 2 * tol * (2 + 2 * math.log(vocab))).all()
    ids = torch.sort(xd, dim=1, descending=True, stable=True).indices[:, :20]
    assert torch.equal(r.top_ids.long(), ids)
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    ref = d.double()[:, None] * (hot - p - p * (logp + h[:, None]))
    off = (r.dlogits.double() - ref).abs()
    bound = d.double().abs()[:, None] * (p * (6 * tol * (2 + logp.abs() + h[:, None])) + 2.0 ** -22 * hot) + UNIT[dtype] * ref.abs() + TINY[dtype]
    assert (off <= bound).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1.0, 1 / 0.7, 3.3])
def test_most_logits_barred_by_any_value(B, dtype, scale):
    import torch
    vocab = 9001
    top = float(torch.finfo(getattr(torch, dtype)).max)
    x = logits(6, vocab, dtype, 12)
    g = torch.Generator(device="cuda").manual_seed(3)
    keep = torch.randperm(vocab, generator=g, device="cuda")[:40]
    barred = torch.ones(vocab, dtype=torch.bool, device="cuda")
    barred[keep] = False
    for row, value in enumerate((-math.inf, -top, -1e10, -3e13, -math.inf, -1e9)):
        x[row, barred] = max(value, -top) if math.isfinite(value) else value
    x[4, keep[5:]] = -math.inf     # fewer are left than alternatives are asked for
    compare(B, x, [int(v) for v in keep[:6]], scale=scale, k=32)


@pytest.mark.parametrize("scale", [0.3, 1.0, 1.7])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_one_large_maximum(B, scale, sign):
    import torch
    x = logits(24, 2000, "float32", 14)
    for row in range(24):   # (the rounding of scale x is then larger than what the other logits differ by)
        x[row] += sign * 3e7 * 1.37 ** row
    compare(B, x, list(range(24)), scale=scale, k=2, weights=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_alternatives_of_equal_and_rising_rows(B, dtype):
    import torch
    vocab = 20000
    x = torch.zeros(4, vocab, device="cuda")
    x[1, 1::2] = 1.0
    x[2] = torch.arange(vocab, device="cuda") // 64 / 64.0
    x[3] = x[2].flip(0)
    compare(B, x.to(getattr(torch, dtype)), [0, 1, 2, 3], k=32, weights=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1, 3, 32, 50, 129, 1000, 2600])
def test_nan_at_the_first_token_and_rows_of_nothing_else(B, dtype, vocab):
    x = logits(4, vocab, dtype, vocab + 1)
    x[0, 0] = math.nan
    x[1] = math.nan
    x[2, 0] = math.nan
    x[2, vocab - 1] = math.inf
    for k in {1, min(vocab, 5), min(vocab, 32)}:     # vocab itself where it is small
        for t in ([0, vocab - 1, 0, vocab // 2], None):
            r = compare(B, x, t, k=k, weights=False)
            assert r.top_ids[1].tolist() == list(range(k)) and r.top_ids[0, 0] == 0
            assert int(r.top_ids.min()) == 0 and int(r.top_ids.max()) < vocab


def test_the_longest_vocabulary(B):
    import torch
    vocab = 2 ** 31 - 1
    buf = torch.zeros(vocab + 8, dtype=torch.bfloat16, device="cuda")
    for shift in (0, 5):
        x = buf[shift:shift + vocab][None]
        buf.zero_()
        x[0, -1], x[0, -2], x[0, 7] = 30.0, 29.0, 28.0
        t, d = torch.tensor([vocab - 1], device="cuda"), torch.ones(1, device="cuda")
        r = B.adapt_token_logprobs(x, t, n_top=3, d_logprob=d, dlogits=x)
        assert r.top_ids.tolist() == [[vocab - 1, vocab - 2, 7]]
        total = vocab - 3 + sum(math.exp(v) for v in (28, 29, 30))
        # a CTA's 256 threads and two chains sum a 16th of the zeros: 2^18 terms each, then chains of 512
        tol = 2.0 ** -21 * (2 + 30) + (2 ** 18 + 512) * 2.0 ** -24
        assert abs(float(r.lse) - math.log(total)) <= tol
        assert abs(float(r.logprob) - (30 - math.log(total))) <= 2 * tol
        want = {vocab - 1: 1 - math.exp(30) / total, vocab - 2: -math.exp(29) / total, 7: -math.exp(28) / total, 0: -1 / total,
                vocab // 2: -1 / total, vocab - 3: -1 / total}
        for j, g in want.items():
            assert abs(float(x[0, j]) - g) <= (2.0 ** -8 + 4 * tol) * abs(g) + 2 * tol * (j == vocab - 1), j
        assert (buf[:shift] == 0).all() and (buf[shift + vocab:] == 0).all()      # nothing beside the row is written


@pytest.mark.parametrize("vocab", [50, 1000, 2600, 20000])
def test_scales_at_the_end_of_the_range(B, vocab):
    for scale in (2.0 ** 127, float(np.float32(3.4e38)), 2.0 ** 120, 2.0 ** -120, 2.0 ** -126):
        x = logits(4, vocab, "float32", vocab)
        x *= 1 / scale if scale > 1 else 1.0        # z of order 3, or next to nothing
        x[1, ::3] = -math.inf
        x[2] -= 2 / scale if scale > 1 else 0.0
        r = compare(B, x, [0, 1, 2, 3], scale=scale, k=3, weights=False)
        assert r.lse.isfinite().all() and r.entropy.isfinite().all()
