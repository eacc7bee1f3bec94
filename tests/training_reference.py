"""Plain implementations in 64 bits (numpy, CPU) of the training-step operators, written from their
definitions.  Inputs are arrays of float64 that hold the exact values of the operators' inputs."""
import math

import numpy as np

C1, C2, C3 = 0x9E3779B97F4A7C15, 0x6A09E667F3BCC909, 0xBB67AE8584CAA73B
DOMAIN = 0xA54FF53A5F1D36F1
M64 = (1 << 64) - 1


def dropout_bits(e, seed, layer):
    """The 32 bits of element number e, in Python integers."""
    z = ((seed ^ DOMAIN ^ ((layer + 1) * C1)) + (e >> 1) * C2) & M64
    z ^= z >> 32
    z = (z * C1) & M64
    z ^= z >> 29
    z = (z * C3) & M64
    z ^= z >> 32
    return z & 0xFFFFFFFF if e & 1 else z >> 32


def dropout_keep(n, p, seed, layer, index_base=0):
    threshold = round(p * 2.0 ** 32)
    return np.array([dropout_bits((index_base + i) & M64, seed, layer) >= threshold for i in range(n)], dtype=bool)


def scaled(x, scale):
    """scale * x, which the operators form in fp32: beyond its range it is infinite."""
    z = x * scale
    z[np.abs(z) > float(np.finfo(np.float32).max)] *= np.inf
    return z


def logprobs(x, targets, scale, k):
    """dict of logprob, entropy, lse, top_ids, top_logprobs of rows of logits."""
    rows, vocab = x.shape
    out = {"logprob": np.zeros(rows), "entropy": np.zeros(rows), "lse": np.zeros(rows),
           "top_ids": np.full((rows, k), -1, dtype=np.int64), "top_logprobs": np.zeros((rows, k))}
    for r in range(rows):
        t = None if targets is None else int(targets[r])
        if t is not None and t < 0:
            continue
        z = scaled(x[r], scale)
        order = sorted(range(vocab), key=lambda j: (0 if math.isnan(x[r, j]) else 1, 0 if math.isnan(x[r, j]) else -x[r, j], j))
        out["top_ids"][r] = order[:k]
        if np.isnan(z).any() or (z == np.inf).any():
            lse = h = math.nan
        elif (z == -np.inf).all():
            lse, h = -math.inf, 0.0
        else:
            m = z.max()
            e = np.exp(z - m)
            lse = m + math.log(e.sum())
            p = np.exp(z - lse)
            h = -sum(pi * (zi - lse) for pi, zi in zip(p, z) if pi > 0)
        out["lse"][r], out["entropy"][r] = lse, h
        for i, j in enumerate(order[:k]):
            out["top_logprobs"][r, i] = -math.inf if lse == -math.inf else z[j] - lse
        if t is not None:
            out["logprob"][r] = math.nan if t >= vocab else (-math.inf if lse == -math.inf else z[t] - lse)
    return out


def logprobs_gradient(x, targets, scale, lse, entropy, dlp, dh):
    rows, vocab = x.shape
    g = np.zeros_like(x)
    for r in range(rows):
        t = None if targets is None else int(targets[r])
        if t is not None and t < 0:
            continue
        if lse[r] == -math.inf:
            continue
        logp = scaled(x[r], scale) - lse[r]
        p = np.exp(logp)
        if dlp is not None:
            g[r] -= dlp[r] * p
            if t < vocab:
                g[r, t] += dlp[r]
            else:
                g[r] = math.nan
        if dh is not None:
            some = p > 0
            g[r, some] -= dh[r] * p[some] * (logp[some] + entropy[r])
        if math.isnan(lse[r]):
            g[r] = math.nan
        g[r] *= scale
    return g


def scan(x, gate, h0, lengths, reset, sigmoid, dy=None, dh_last=None):
    """(y, h_last, states before each step) and, with dy, (dx, dgate, dh0) too."""
    B, T, D = x.shape
    group = D // gate.shape[2] if D else 1
    g = np.repeat(gate, group, axis=2)
    with np.errstate(over="ignore"):
        a = 1 / (1 + np.exp(-g)) if sigmoid else g
        c = 1 / (1 + np.exp(g)) if sigmoid else np.ones_like(g)
    h = np.zeros((B, D)) if h0 is None else h0.copy()
    n = [T if lengths is None else max(0, min(T, int(lengths[b]))) for b in range(B)]
    y, before = np.zeros((B, T, D)), np.zeros((B, T, D))
    for b in range(B):
        for t in range(n[b]):
            cut = reset is not None and reset[b, t]
            before[b, t] = 0 if cut else h[b]
            h[b] = (0 if cut else a[b, t] * h[b]) + c[b, t] * x[b, t]
            y[b, t] = h[b]
    if dy is None:
        return y, h, before
    flow = np.zeros((B, D)) if dh_last is None else dh_last.copy()
    dx, dg = np.zeros((B, T, D)), np.zeros((B, T, D))
    for b in range(B):
        for t in reversed(range(n[b])):
            dh = dy[b, t] + flow[b]
            dx[b, t] = dh * c[b, t]
            dg[b, t] = dh * (before[b, t] - x[b, t]) * a[b, t] * c[b, t] if sigmoid else dh * before[b, t]
            flow[b] = 0 if reset is not None and reset[b, t] else a[b, t] * dh
    return (y, h, before), (dx, dg.reshape(B, T, D // group, group).sum(3), flow)
