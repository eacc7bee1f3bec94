"""Plain implementations in 64 bits (torch, any device) of the operators around a language model's layers,
written from their definitions, with the bounds of what fp32 arithmetic in any order may add.

u = 2^-24 is half a step of fp32."""
import math

import torch

U = 2.0 ** -24
TINY = 2.0 ** -100
NONE, RMS, LAYER = 0, 1, 2


def half_step(v, dtype):
    """How far the rounding of v to dtype may go: half a step, relative, and in the subnormal range absolute."""
    f = torch.finfo(dtype)
    return v.abs() * (f.eps / 2) + f.tiny * f.eps / 2


def within(got, want, tol):
    """Whether got is within tol of want, with NaN and infinities where they are."""
    got, want = got.double(), want.double()
    same = (got == want) | (got.isnan() & want.isnan())
    return bool((same | ((got - want).abs() <= tol)).all())


# ---- embedding -----------------------------------------------------------------------------------

def embedding(table, ids, scale):
    vocab = table.shape[0]
    out = table.double()[ids.clamp(0, vocab - 1)] * scale
    out[ids < 0] = 0.0
    out[ids >= vocab] = math.nan
    return out


def embedding_gradient(dy, ids, vocab, scale):
    """(gradient, bound of the error of its fp32 sums): a sum of m terms is m additions and two products."""
    live = (ids >= 0) & (ids < vocab)
    dy, ids = dy.double()[live], ids[live]
    zeros = lambda: torch.zeros((vocab, dy.shape[1]), dtype=torch.float64, device=dy.device)  # noqa: E731
    count = torch.zeros(vocab, dtype=torch.float64, device=dy.device).index_add_(0, ids, torch.ones_like(ids, dtype=torch.float64))
    size = zeros().index_add_(0, ids, dy.abs())
    return zeros().index_add_(0, ids, dy) * scale, (count[:, None] + 3) * U * size * abs(scale)


# ---- 8-bit codes ---------------------------------------------------------------------------------

def int8_rows(x):
    """Codes (as float64) and scales (float32)."""
    x = x.double()
    if x.shape[1] == 0:
        largest = torch.zeros(x.shape[0], dtype=torch.float64, device=x.device)
    else:
        largest = x.abs().amax(1)
    bad = ~torch.isfinite(largest) | x.isnan().any(1)
    largest = torch.where(bad, 1.0, largest.clamp(min=TINY))
    inverse = (127.0 / largest).float().double()     # both exact in fp32: rounded as one fp32 division is
    codes = torch.round(torch.where(bad[:, None], 0.0, x) * inverse[:, None])
    scales = (largest / 127.0).float()
    scales[bad] = math.nan
    return codes, scales


def int8_linear(codes, x_scales, w, w_scales, bias):
    """(y, bound): the sum is exact, its conversion, two products and the bias round once each."""
    total = codes.double() @ w.double().t()
    y = total * x_scales.double().reshape(-1, 1) * w_scales.double().reshape(1, -1)
    tol = 3.01 * U * y.abs()
    if bias is not None:
        y = y + bias.double()
        tol = tol + U * y.abs()
    return y, tol + 2.0 ** -140


# ---- norms around a block ------------------------------------------------------------------------

def _statistics(v, kind, eps):
    mean = v.mean(1, keepdim=True) if kind == LAYER else torch.zeros_like(v[:, :1])
    return mean, 1 / ((v - mean).square().mean(1, keepdim=True) + eps).sqrt()


class Norms:
    """Forward and, with gradients given, backward pass; tolerances of fp32 arithmetic beside them.

    Bounds.  A sum of a row's dim terms has at most dim / 32 additions one after the other and 32 joins; with the
    roundings around it (products, the square root's reciprocal to 2 ulp, the exponential to 2 ulp and |gate| of
    its argument's steps) everything computed from a row is off by at most c = 8 (dim / 32 + |gate| + 48) u of
    what its terms are in magnitude, where a norm multiplies what its input was off by: `grow` is the
    largest of the terms of its input by its deviation (1 where nothing cancels).  The gradients are bounded by the same
    formulas with every term's magnitude.

    A gate beyond +-87.3 has e^-|gate| < 2^-126, the least normal number of fp32: what is below has no relative
    precision (it may be held in steps of 2^-149 or be 0), so the gate and its slope are off by up to 2^-126 besides; `open_size`
    and `slope_size` are their magnitudes with 2^-126 / c added, which c takes back."""

    def __init__(self, block, residual, gate, wa, wb, after, before, sigmoid, scale, residual_scale, eps, d_y=None, d_normed=None):
        block = block.double()
        rows, dim = block.shape
        one = torch.ones(dim, dtype=torch.float64, device=block.device)
        wa, wb = (one if w is None else w.double() for w in (wa, wb))
        mean_a, r_a = _statistics(block, after, eps) if after != NONE else (0.0, 1.0)
        hat = (block - mean_a) * r_a if after != NONE else block
        value = hat * wa if after != NONE else hat
        raw = None if gate is None else gate.double().expand(rows, dim)
        open_ = torch.ones_like(block) if gate is None else torch.sigmoid(raw) if sigmoid else raw
        slope = torch.sigmoid(raw) * torch.sigmoid(-raw) if gate is not None and sigmoid else torch.ones_like(block)
        steepest = 0.0 if raw is None or not sigmoid else float(raw.abs().max())
        c = 8 * (dim / 32 + steepest + 48) * U
        open_size, slope_size = open_.abs() + 2.0 ** -126 / c, slope + 2.0 ** -126 / c
        y = value * open_ * scale
        terms = ((block.abs() + abs(mean_a)) * r_a * wa.abs() if after != NONE else block.abs()) * open_size * abs(scale)
        if residual is not None:
            y = y + residual.double() * residual_scale
            terms = terms + residual.double().abs() * abs(residual_scale)
        grow_a = 1 + (float(((block.abs() + abs(mean_a)) * r_a).max()) if after != NONE else 0.0)
        self.y, self.y_tol = y, c * (terms + (value * open_ * scale).abs() * grow_a)
        grow = torch.ones_like(y[:, :1])
        if before != NONE:
            mean_b, r_b = _statistics(y, before, eps)
            y_hat = (y - mean_b) * r_b
            grow = 1 + ((terms + abs(mean_b)).amax(1, keepdim=True)) * r_b * grow_a
            self.normed = y_hat * wb
            self.normed_tol = c * grow * (1 + y_hat.abs()) * wb.abs()
        if d_y is None and d_normed is None:
            return
        d = torch.zeros_like(y) if d_y is None else d_y.double()
        size = d.abs()
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        if d_normed is not None:
            dn = d_normed.double()
            self.d_weight_before = (dn * y_hat).sum(0)
            self.d_weight_before_tol = ((c * grow + (rows + 8) * U) * dn.abs() * (1 + y_hat.abs())).sum(0)
            g = dn * wb
            d = d + r_b * (g - y_hat * mean(g * y_hat) - (mean(g) if before == LAYER else 0.0))
            size = size + grow * r_b * (g.abs() + (1 + y_hat.abs()) * mean(g.abs() * (1 + y_hat.abs())) + mean(g.abs()))
        self.d_residual, self.d_residual_tol = d * residual_scale, c * size * abs(residual_scale)
        d, size = d * scale, size * abs(scale)
        if gate is not None:
            self.d_gate = d * value * slope
            self.d_gate_tol = c * grow_a * size * ((1 + hat.abs()) * wa.abs() if after != NONE else value.abs()) * slope_size
            if gate.dim() == 1:
                self.d_gate_tol = (self.d_gate_tol + (rows + 8) * U * self.d_gate.abs()).sum(0)
                self.d_gate = self.d_gate.sum(0)
        d, size = d * open_, size * open_size
        if after != NONE:
            self.d_weight_after = (d * hat).sum(0)
            self.d_weight_after_tol = ((c * grow_a + (rows + 8) * U) * size * (1 + hat.abs())).sum(0)
            g, g_size = d * wa, size * wa.abs()
            d = r_a * (g - hat * mean(g * hat) - (mean(g) if after == LAYER else 0.0))
            size = grow_a * r_a * (g_size + (1 + hat.abs()) * mean(g_size * (1 + hat.abs())) + mean(g_size))
        self.d_block, self.d_block_tol = d, c * size
