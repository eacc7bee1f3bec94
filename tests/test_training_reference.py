"""The 64-bit reference of the training-step operators: hand-worked values, and its gradients against
central differences of its own forward pass.  CPU only."""
import math

import numpy as np
import pytest

from tests import training_reference as R


def test_dropout_bits_match_a_second_formulation():
    # the same hash in wrapping numpy arithmetic
    with np.errstate(over="ignore"):
        for seed, layer in ((0, 0), (12345678901234567, 7), (2 ** 64 - 1, -1)):
            j = np.arange(50, dtype=np.uint64)
            z = j * np.uint64(R.C2) + np.uint64((seed ^ R.DOMAIN ^ ((layer + 1) * R.C1)) & R.M64)
            z ^= z >> np.uint64(32)
            z *= np.uint64(R.C1)
            z ^= z >> np.uint64(29)
            z *= np.uint64(R.C3)
            z ^= z >> np.uint64(32)
            want = np.stack([z >> np.uint64(32), z & np.uint64(0xFFFFFFFF)], 1).reshape(-1)
            got = np.array([R.dropout_bits(e, seed, layer) for e in range(100)], dtype=np.uint64)
            assert np.array_equal(got, want)


def test_dropout_bits_are_uniform_and_independent_of_neighbours():
    n = 40000
    for seed, layer in ((1, 0), (99, 5)):
        u = np.array([R.dropout_bits(e, seed, layer) for e in range(n)], dtype=np.float64) / 2 ** 32
        assert abs(u.mean() - 0.5) < 5 * math.sqrt(1 / 12 / n)
        counts = np.histogram(u, bins=64, range=(0, 1))[0]
        chi2 = ((counts - n / 64) ** 2 / (n / 64)).sum()
        assert chi2 < 63 + 5 * math.sqrt(2 * 63)
        for lag in (1, 2, 3):
            r = np.corrcoef(u[:-lag], u[lag:])[0, 1]
            assert abs(r) < 5 / math.sqrt(n)


def test_logprobs_by_hand():
    x = np.array([[0.0, 0.0, 0.0, 0.0], [0.0, math.log(3), -math.inf, -math.inf], [-math.inf] * 4,
                  [1.0, 2.0, 2.0, math.nan]])
    o = R.logprobs(x, np.array([1, 1, 2, -1]), 1.0, 3)
    assert np.allclose(o["logprob"], [-math.log(4), math.log(0.75), -math.inf, 0.0])
    assert np.allclose(o["entropy"], [math.log(4), -0.25 * math.log(0.25) - 0.75 * math.log(0.75), 0.0, 0.0])
    assert o["top_ids"].tolist() == [[0, 1, 2], [1, 0, 2], [0, 1, 2], [-1, -1, -1]]
    o = R.logprobs(x[3:], None, 1.0, 3)
    assert o["top_ids"].tolist() == [[3, 1, 2]] and math.isnan(o["lse"][0])


def test_logprobs_gradient_against_differences():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 9)) * 2
    x[1, 3] = -math.inf
    t, scale = np.array([2, 5, -1]), 1.4
    dlp, dh = rng.standard_normal(3), rng.standard_normal(3)

    def value(x):
        o = R.logprobs(x, t, scale, 0)
        return (o["logprob"] * dlp + o["entropy"] * dh).sum()

    o = R.logprobs(x, t, scale, 0)
    g = R.logprobs_gradient(x, t, scale, o["lse"], o["entropy"], dlp, dh)
    eps = 1e-5
    for r in range(3):
        for j in range(9):
            if math.isinf(x[r, j]):
                assert g[r, j] == 0
                continue
            a, b = x.copy(), x.copy()
            a[r, j] += eps
            b[r, j] -= eps
            assert abs((value(a) - value(b)) / (2 * eps) - g[r, j]) < 1e-8


def test_scan_by_hand():
    x = np.array([[[1.0], [2.0], [4.0], [8.0]]])
    gate = np.array([[[0.5], [0.5], [0.25], [3.0]]])
    y, h, before = R.scan(x, gate, np.array([[2.0]]), None, None, False)
    assert y.ravel().tolist() == [2.0, 3.0, 4.75, 22.25] and h[0, 0] == 22.25
    assert before.ravel().tolist() == [2.0, 2.0, 3.0, 4.75]
    y, h, _ = R.scan(x, gate, np.array([[math.inf]]), np.array([3]), np.array([[1, 0, 1, 0]], dtype=np.uint8), False)
    assert y.ravel().tolist() == [1.0, 2.5, 4.0, 0.0] and h[0, 0] == 4.0
    y, h, _ = R.scan(x, np.zeros_like(gate), None, None, None, True)
    assert y.ravel().tolist() == [0.5, 1.25, 2.625, 5.3125]
    y, h, _ = R.scan(x, gate, np.array([[7.0]]), np.array([0]), None, True)
    assert not y.any() and h[0, 0] == 7.0


@pytest.mark.parametrize("sigmoid", [False, True])
def test_scan_gradient_against_differences(sigmoid):
    rng = np.random.default_rng(1)
    B, T, D, G = 2, 6, 4, 2
    x, gate, h0 = rng.standard_normal((B, T, D)), rng.standard_normal((B, T, G)), rng.standard_normal((B, D))
    lengths, reset = np.array([6, 4]), np.zeros((B, T), dtype=np.uint8)
    reset[0, 3] = reset[1, 0] = reset[1, 5] = 1
    dy, dl = rng.standard_normal((B, T, D)), rng.standard_normal((B, D))

    def value(x, gate, h0):
        y, h, _ = R.scan(x, gate, h0, lengths, reset, sigmoid)
        return (y * dy).sum() + (h * dl).sum()

    _, grads = R.scan(x, gate, h0, lengths, reset, sigmoid, dy, dl)
    eps = 1e-5
    for k, (v, g) in enumerate(zip((x, gate, h0), grads)):
        for i in np.ndindex(v.shape):
            args = [[x, gate, h0], [x, gate, h0]]
            for s, a in zip((1, -1), args):
                a[k] = v.copy()
                a[k][i] += s * eps
            d = (value(*args[0]) - value(*args[1])) / (2 * eps)
            assert abs(d - g[i]) < 1e-7, (k, i)
