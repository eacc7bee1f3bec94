"""Cases and plain forms of the operators around a language model's layers: the product with 8-bit
codes, the token embedding with its gradient, and the norms before and after a block.

With ``own`` false, ``run`` computes an operator from elementary torch operations in 32 bits (64 for
the rounding to codes, where values lie next to a border); with ``own`` true it makes the calls that a
user makes of this package.  ``exact`` gives the same outputs in 64 bits from the definitions.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
_TINY = 2.0 ** -100     # a row whose largest magnitude is smaller is quantised as if it were this
_EPS = 1e-6


def listed():
    return [
        # one decoded token through a square layer, its activations quantised within the call
        {"name": "int8_one_token", "op": "int8", "rows": 1, "k": 4096, "n": 4096, "x": "bf16", "y": "bf16",
         "bias": False, "tensor_scale": False},
        # one token for each of 64 running requests through a widening layer
        {"name": "int8_batch", "op": "int8", "rows": 64, "k": 4096, "n": 16384, "x": "bf16", "y": "bf16",
         "bias": False, "tensor_scale": False},
        # prompt processing: 8192 tokens through the same layer
        {"name": "int8_prompt", "op": "int8", "rows": 8192, "k": 4096, "n": 16384, "x": "bf16", "y": "bf16",
         "bias": False, "tensor_scale": False},
        # activations that are codes already, fixed-point weights (one scale for the layer), a bias, odd sizes
        {"name": "int8_ragged", "op": "int8", "rows": 777, "k": 1001, "n": 1531, "x": "i8", "y": "f32",
         "bias": True, "tensor_scale": True},
        # the tokens that 256 running requests decoded last, out of a large table
        {"name": "embed_tokens", "op": "embed", "tokens": 256, "vocab": 131072, "dim": 4096, "dtype": "bf16",
         "grad": "bf16", "padded": False, "train": False},
        # a training step's tokens, frequent and rare ones, and the gradient of the whole table
        {"name": "embed_train", "op": "embed", "tokens": 16384, "vocab": 65536, "dim": 2048, "dtype": "bf16",
         "grad": "bf16", "padded": False, "train": True},
        # the vocabulary of the recurrent example: every row of the table occurs many times; fp32 gradient
        {"name": "embed_bytes", "op": "embed", "tokens": 65536, "vocab": 512, "dim": 1024, "dtype": "bf16",
         "grad": "f32", "padded": False, "train": True},
        # a padded batch of an odd width
        {"name": "embed_ragged", "op": "embed", "tokens": 4099, "vocab": 50257, "dim": 1001, "dtype": "f16",
         "grad": "f16", "padded": True, "train": True},
        # one token for each of 64 requests between two blocks
        {"name": "norm_step", "op": "norm", "rows": 64, "dim": 4096, "dtype": "bf16", "after": "rms",
         "before": "rms", "gate": "sigmoid", "residual": True, "train": False},
        # a training step between two blocks, both ways
        {"name": "norm_train", "op": "norm", "rows": 16384, "dim": 4096, "dtype": "bf16", "after": "rms",
         "before": "rms", "gate": "sigmoid", "residual": True, "train": True},
        # a norm alone before a block, fp32, both ways
        {"name": "norm_before", "op": "norm", "rows": 32768, "dim": 1024, "dtype": "f32", "after": "none",
         "before": "rms", "gate": "none", "residual": False, "train": True},
        # norms with a mean, one gate for all rows, odd sizes, both ways
        {"name": "norm_ragged", "op": "norm", "rows": 4099, "dim": 1001, "dtype": "f16", "after": "layer",
         "before": "layer", "gate": "shared", "residual": True, "train": True},
    ]


def _between(rng, lo, hi):
    """A whole number in lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["int8", "embed", "norm"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "int8":
        k = _between(rng, 16, 16384)
        n = _between(rng, 16, min(32768, (1 << 27) // k))
        if rng.random() < 0.6:      # most layers are multiples of 64 wide
            k, n = -(-k // 64) * 64, -(-n // 64) * 64
        rows = _between(rng, 1, max(1, min(8192, (1 << 38) // (k * n))))
        return {"op": op, "rows": rows, "k": k, "n": n, "x": rng.choice(["bf16", "bf16", "f16", "f32", "i8"]), "y": dtype,
                "bias": rng.random() < 0.3, "tensor_scale": rng.random() < 0.3}
    if op == "embed":
        dim = _between(rng, 1, 8192)
        if rng.random() < 0.6:
            dim = -(-dim // 64) * 64
        vocab = _between(rng, 10, min(200000, (1 << 27) // dim))
        return {"op": op, "tokens": _between(rng, 1, min(131072, (1 << 26) // dim)), "vocab": vocab, "dim": dim, "dtype": dtype,
                "grad": rng.choice([dtype, "f32"]), "padded": rng.random() < 0.4, "train": rng.random() < 0.7}
    dim = _between(rng, 16, 16384)
    if rng.random() < 0.6:
        dim = -(-dim // 64) * 64
    after, before = rng.choice(["none", "rms", "layer"]), rng.choice(["none", "rms", "layer"])
    if after == before == "none":
        before = "rms"
    return {"op": op, "rows": _between(rng, 1, min(65536, (1 << 26) // dim)), "dim": dim, "dtype": dtype, "after": after,
            "before": before, "gate": rng.choice(["none", "sigmoid", "value", "shared"]), "residual": rng.random() < 0.7,
            "train": rng.random() < 0.6}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = {"case": case}
    if case["op"] == "int8":
        rows, k, n = case["rows"], case["k"], case["n"]
        w = normal(n, k, scale=k ** -0.5)
        if case["tensor_scale"]:    # fixed-point codes <8, FL>: the largest FL that holds four deviations
            fl = math.floor(math.log2(127 / (4 * k ** -0.5)))
            s["ws"] = torch.full((1,), 2.0 ** -fl, device="cuda")
        else:                       # a scale for each channel
            s["ws"] = w.abs().amax(1).clamp(min=_TINY) / 127
        s["w"] = torch.round(w / s["ws"][:, None]).clamp(-128, 127).to(torch.int8)
        x = normal(rows, k)
        x[:, torch.randperm(k, generator=g, device="cuda")[:max(1, k // 256)]] *= 12     # channels that stand out
        if case["x"] == "i8":
            s["xs"] = x.abs().amax(1) / 127
            x = torch.round(x / s["xs"][:, None]).clamp(-127, 127).to(torch.int8)
        else:
            x = x.to(_DTYPES[case["x"]])
        s["x"] = x
        s["bias"] = normal(n) if case["bias"] else None
        return s
    dt = _DTYPES[case["dtype"]]
    if case["op"] == "embed":
        n, vocab, dim = case["tokens"], case["vocab"], case["dim"]
        s["table"] = normal(vocab, dim, scale=dim ** -0.5, dtype=dt)
        # the frequency of a token falls with its rank; ranks are spread over the table
        rank = torch.pow(float(vocab), torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).long().sub_(1).clamp_(0, vocab - 1)
        ids = torch.randperm(vocab, generator=g, device="cuda")[rank]
        if case["padded"]:
            ids = torch.where(torch.rand(n, generator=g, device="cuda") < 1 / 16, torch.full_like(ids, -1), ids)
        s["ids"], s["scale"] = ids, math.sqrt(dim)
        if case["train"]:
            s["dy"] = normal(n, dim, dtype=dt)
        return s
    rows, dim = case["rows"], case["dim"]
    s["block"] = normal(rows, dim, scale=0.7, shift=0.05, dtype=dt)
    s["residual"] = normal(rows, dim, scale=2.0, dtype=dt) if case["residual"] else None
    s["gate"] = {"none": lambda: None, "sigmoid": lambda: normal(rows, dim, scale=1.5, dtype=dt),
                 "value": lambda: normal(rows, dim, scale=0.5, shift=1.0, dtype=dt),
                 "shared": lambda: normal(dim, scale=0.2, shift=0.5)}[case["gate"]]()
    s["wa"] = normal(dim, scale=0.2, shift=1.0) if case["after"] != "none" else None
    s["wb"] = normal(dim, scale=0.2, shift=1.0) if case["before"] != "none" else None
    s["scale"], s["residual_scale"] = 0.5, 1.25
    if case["train"]:
        s["dy"] = normal(rows, dim, dtype=dt) if _has_sum(case) else None
        s["dn"] = normal(rows, dim, dtype=dt) if case["before"] != "none" else None
    return s


def _has_sum(case):
    """Whether there is anything between the block's output and the norm before the next one."""
    return case["residual"] or case["gate"] != "none" or case["after"] != "none"


def work(case):
    if case["op"] == "int8":
        rows, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": rows * k * _BYTES[case["x"]] + n * k + rows * n * _BYTES[case["y"]]
                + 4 * ((rows if case["x"] == "i8" else 0) + (1 if case["tensor_scale"] else n) + (n if case["bias"] else 0)),
                "flops": 2 * rows * k * n}
    e = _BYTES[case["dtype"]]
    if case["op"] == "embed":
        n, vocab, dim = case["tokens"], case["vocab"], case["dim"]
        rows_read = vocab * (1 - (1 - 1 / vocab) ** n) if case["vocab"] < n else n
        b = 8 * n + min(n, rows_read) * dim * e + n * dim * e
        if case["train"]:
            b += n * dim * e + vocab * dim * _BYTES[case["grad"]]
        return {"bytes": b, "flops": n * dim * (2 if case["train"] else 1)}
    m = case["rows"] * case["dim"]
    each, summed, normed = case["gate"] in ("sigmoid", "value"), _has_sum(case), case["before"] != "none"
    tensors = 1 + case["residual"] + each + summed + normed
    if case["train"]:
        tensors += summed + normed + 1 + case["residual"] + each
    return {"bytes": m * e * tensors, "flops": m * (30 if case["train"] else 12)}


def run(state):
    return {"int8": _run_int8, "embed": _run_embed, "norm": _run_norm}[state["case"]["op"]](state)


def exact(case, seed):
    s = prepare(case, seed)
    return {"int8": _exact_int8, "embed": _exact_embed, "norm": _exact_norm}[case["op"]](s)


# ---- product with 8-bit codes --------------------------------------------------------------------

def _plain_codes(x):
    """Codes and scales of the rows: code = x (127 / largest) to the nearest, the quotient in fp32 and the
    product unrounded; scale = largest / 127."""
    largest = x.float().abs().amax(1).clamp(min=_TINY)
    inverse = torch.full_like(largest, 127.0) / largest     # (127 / largest would multiply by a reciprocal)
    codes = torch.round(x.double() * inverse.double()[:, None]).clamp(-127, 127)
    return codes.float(), largest / 127


def _run_int8(s):
    case = s["case"]
    if own:
        from paper_2107_13490_b200 import binding as B
        return B.adapt_int8_linear(s["x"], s["w"], s["ws"], x_scales=s.get("xs"), bias=s["bias"], dtype=_DTYPES[case["y"]])
    codes, scales = (s["x"].float(), s["xs"]) if case["x"] == "i8" else _plain_codes(s["x"])
    y = (codes @ s["w"].float().t()) * scales[:, None] * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(_DTYPES[case["y"]])


def _exact_int8(s):
    x = s["x"].double()
    if s["case"]["x"] == "i8":
        scales = s["xs"].double()
    else:
        largest = x.abs().max(1).values.clamp(min=_TINY)
        # fp32 by definition: rounding the quotient of two fp32 numbers in 64 bits once more is the same
        inverse = torch.div(torch.tensor(127.0, dtype=torch.float64, device=x.device).expand_as(largest), largest).float().double()
        x, scales = torch.round(x * inverse[:, None]), largest / 127
    y = torch.einsum("rk,nk->rn", x, s["w"].double()) * torch.outer(scales, s["ws"].double().expand(s["w"].shape[0]))
    return y if s["bias"] is None else y + s["bias"].double()


# ---- token embedding -----------------------------------------------------------------------------

def _run_embed(s):
    case, ids, scale = s["case"], s["ids"], s["scale"]
    grad = _DTYPES[case["grad"]]
    if own:
        from paper_2107_13490_b200 import binding as B
        out = {"y": B.adapt_embedding(s["table"], ids, scale=scale)}
        if case["train"]:
            out["dtable"] = B.adapt_embedding_backward(s["dy"], ids, case["vocab"], scale=scale, dtype=grad)
        return out
    live = (ids >= 0)[:, None]
    at = ids.clamp(min=0)
    out = {"y": torch.where(live, s["table"][at].float() * scale, 0.0).to(s["table"].dtype)}
    if case["train"]:
        total = torch.zeros((case["vocab"], case["dim"]), device=ids.device)
        total.index_add_(0, at, torch.where(live, s["dy"].float(), 0.0))
        out["dtable"] = (total * scale).to(grad)
    return out


def _exact_embed(s):
    case, ids, scale = s["case"], s["ids"], s["scale"]
    known = torch.nonzero(ids >= 0)[:, 0]
    y = torch.zeros((case["tokens"], case["dim"]), dtype=torch.float64, device=ids.device)
    y[known] = torch.index_select(s["table"], 0, ids[known]).double() * scale
    out = {"y": y}
    if case["train"]:
        total = torch.zeros((case["vocab"], case["dim"]), dtype=torch.float64, device=ids.device)
        out["dtable"] = total.index_put_((ids[known],), s["dy"][known].double() * scale, accumulate=True)
    return out


# ---- norms around a block ------------------------------------------------------------------------

def _normed(v, kind):
    """(v normalised, 1 / deviation) of the rows, from elementary operations."""
    if kind == "layer":
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    rstd = 1 / torch.sqrt((v * v).sum(1, keepdim=True) / v.shape[1] + _EPS)
    return v * rstd, rstd


def _norm_gradient(d, hat, rstd, kind):
    """The gradient of v from that of its normalised form."""
    d = d - hat * ((d * hat).sum(1, keepdim=True) / d.shape[1]) - (d.sum(1, keepdim=True) / d.shape[1] if kind == "layer" else 0.0)
    return d * rstd


def _run_norm(s):
    case = s["case"]
    if own:
        return _own_norm(s)
    dt = s["block"].dtype
    block, gate = s["block"].float(), None if s["gate"] is None else s["gate"].float()
    after, before = case["after"], case["before"]
    hat, rstd = _normed(block, after) if after != "none" else (block, None)
    value = hat * s["wa"] if after != "none" else hat
    open_ = 1.0 if gate is None else 1 / (1 + torch.exp(-gate)) if case["gate"] == "sigmoid" else gate
    y = value * open_ * s["scale"] if _has_sum(case) else value
    if s["residual"] is not None:
        y = y + s["residual"].float() * s["residual_scale"]
    out = {}
    if _has_sum(case):
        out["y"] = y.to(dt)
    if before != "none":
        y_hat, y_rstd = _normed(y, before)
        out["normed"] = (y_hat * s["wb"]).to(dt)
    if not case["train"]:
        return out
    d = 0.0 if s["dy"] is None else s["dy"].float()
    if before != "none":
        dn = s["dn"].float()
        out["d_weight_before"] = (dn * y_hat).sum(0)
        d = d + _norm_gradient(dn * s["wb"], y_hat, y_rstd, before)
    if s["residual"] is not None:
        out["d_residual"] = (d * s["residual_scale"]).to(dt)
    if _has_sum(case):
        d = d * s["scale"]
    if gate is not None:
        d_gate = d * value
        if case["gate"] == "sigmoid":
            d_gate = d_gate * open_ * (1 - open_)
        out["d_gate"] = d_gate.sum(0) if case["gate"] == "shared" else d_gate.to(dt)
        d = d * open_
    if after != "none":
        out["d_weight_after"] = (d * hat).sum(0)
        d = _norm_gradient(d * s["wa"], hat, rstd, after)
    out["d_block"] = d.to(dt)
    return out


def _own_norm(s):
    from paper_2107_13490_b200 import binding as B
    case, kinds = s["case"], {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
    how = dict(residual=s["residual"], gate=s["gate"], weight_after=s["wa"], weight_before=s["wb"],
               after=kinds[case["after"]], before=kinds[case["before"]],
               gate_mode=B.GATE_SIGMOID if case["gate"] == "sigmoid" else B.GATE_VALUE, eps=_EPS)
    if _has_sum(case):
        how.update(scale=s["scale"], residual_scale=s["residual_scale"])
    r = B.adapt_block_norm(s["block"], want_y=_has_sum(case), want_stats=case["train"], **how)
    out = {"y": r.y, "normed": r.normed}
    if case["train"]:
        g = B.adapt_block_norm_backward(s["block"], r.stats, d_y=s["dy"], d_normed=s["dn"], **how)
        out.update(d_block=g.d_block, d_residual=g.d_residual, d_gate=g.d_gate, d_weight_after=g.d_weight_after,
                   d_weight_before=g.d_weight_before)
    return {name: v for name, v in out.items() if v is not None}


def _exact_norm(s):
    """Forward in 64 bits; the gradients by differentiating it."""
    case = s["case"]
    inputs = {"block": s["block"], "residual": s["residual"], "gate": s["gate"], "weight_after": s["wa"], "weight_before": s["wb"]}
    inputs = {name: v.double().requires_grad_(case["train"]) for name, v in inputs.items() if v is not None}

    def norm(v, kind, w):
        if kind == "none":
            return v
        if kind == "layer":
            v = v - v.mean(1, keepdim=True)
        return v / (v.square().mean(1, keepdim=True) + _EPS).sqrt() * w

    with torch.set_grad_enabled(case["train"]):
        y = norm(inputs["block"], case["after"], inputs.get("weight_after"))
        if case["gate"] != "none":
            y = y * (torch.sigmoid(inputs["gate"]) if case["gate"] == "sigmoid" else inputs["gate"])
        if _has_sum(case):
            y = y * s["scale"]
        if case["residual"]:
            y = y + s["residual_scale"] * inputs["residual"]
        normed = norm(y, case["before"], inputs.get("weight_before"))
        out = {}
        if _has_sum(case):
            out["y"] = y.detach()
        if case["before"] != "none":
            out["normed"] = normed.detach()
        if case["train"]:
            total = 0.0
            if s["dy"] is not None:
                total = total + (y * s["dy"].double()).sum()
            if s["dn"] is not None:
                total = total + (normed * s["dn"].double()).sum()
            for name, d in zip(inputs, torch.autograd.grad(total, list(inputs.values()))):
                out["d_" + name] = d
    return out
