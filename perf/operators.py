"""Cases and plain forms of the training-step operators: dropout from a counter, token log
probabilities with entropy and alternatives, and the gated linear recurrence.

With ``own`` false, ``run`` computes an operator from elementary torch operations in 32 bits;
with ``own`` true it makes the calls that a user makes of this package.  ``exact`` gives the same
outputs in 64 bits from the definitions.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_M64 = (1 << 64) - 1


def listed():
    return [
        # one decoded token: log probability of the sampled token, entropy and 8 alternatives
        {"name": "logprobs_one_token", "op": "logprobs", "rows": 1, "vocab": 131072, "dtype": "bf16",
         "top": 8, "temperature": 1.0, "train": "no", "masked": True},
        # a serving batch at temperature 0.7 with 20 alternatives, fp32 logits
        {"name": "logprobs_batch", "op": "logprobs", "rows": 64, "vocab": 32000, "dtype": "f32",
         "top": 20, "temperature": 0.7, "train": "no", "masked": True},
        # the classifier head of the CIFAR networks: 10 classes, batch 128, loss and gradient
        {"name": "logprobs_classes", "op": "logprobs", "rows": 128, "vocab": 10, "dtype": "f32",
         "top": 3, "temperature": 1.0, "train": "loss", "masked": False},
        # the loss of a language model's training step: weights known before, so loss and gradient in one call
        {"name": "logprobs_loss", "op": "logprobs", "rows": 4096, "vocab": 65536, "dtype": "bf16",
         "top": 0, "temperature": 1.0, "train": "loss", "masked": False},
        # policy-gradient style: statistics first, their gradient later; rows of an odd length
        {"name": "logprobs_ragged", "op": "logprobs", "rows": 1531, "vocab": 50257, "dtype": "f16",
         "top": 5, "temperature": 1.0, "train": "later", "masked": True},
        # one token for each of 256 running requests: the recurrence's state in, state out
        {"name": "scan_step", "op": "scan", "batch": 256, "steps": 1, "channels": 4096, "group": 1,
         "dtype": "bf16", "form": "sigmoid", "train": False, "lengths": False, "resets": False, "state": True},
        # a training step's sequence layer, forward and backward
        {"name": "scan_train", "op": "scan", "batch": 8, "steps": 4096, "channels": 2048, "group": 1,
         "dtype": "bf16", "form": "sigmoid", "train": True, "lengths": False, "resets": False, "state": False},
        # one long packed sequence (documents end at resets), prompt processing with the final state
        {"name": "scan_long", "op": "scan", "batch": 1, "steps": 65536, "channels": 1024, "group": 1,
         "dtype": "bf16", "form": "sigmoid", "train": False, "lengths": False, "resets": True, "state": True},
        # ragged batch, gates shared by four channels, given decays, fp32, forward and backward
        {"name": "scan_ragged", "op": "scan", "batch": 5, "steps": 1531, "channels": 1000, "group": 4,
         "dtype": "f32", "form": "value", "train": True, "lengths": True, "resets": True, "state": True},
        # dropout behind the 4096-wide layers of the AlexNet workload, batch 128
        {"name": "dropout_fc", "op": "dropout", "rows": 128, "cols": 4096, "pad": 0, "dtype": "f32",
         "p": 0.5, "residual": False, "train": False},
        # a block's output: dropout and residual sum, forward and backward
        {"name": "dropout_residual", "op": "dropout", "rows": 16384, "cols": 4096, "pad": 0, "dtype": "bf16",
         "p": 0.1, "residual": True, "train": True},
        # an odd slice of a wider buffer
        {"name": "dropout_slice", "op": "dropout", "rows": 4099, "cols": 1001, "pad": 47, "dtype": "f16",
         "p": 0.2, "residual": False, "train": False},
    ]


def _between(rng, lo, hi):
    """A whole number in lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprobs", "scan", "dropout"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "logprobs":
        vocab = _between(rng, 10, 200000)
        rows = _between(rng, 1, max(1, min(16384, (1 << 27) // vocab)))
        return {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype,
                "top": min(vocab, rng.choice([0, 1, 5, 8, 20, 32])), "temperature": rng.choice([1.0, 0.7, 1.3]),
                "train": rng.choice(["no", "loss", "later"]), "masked": rng.random() < 0.5}
    if op == "scan":
        group = rng.choice([1, 1, 1, 2, 8, 64, 128])
        channels = max(1, _between(rng, 64, 8192) // group) * group
        batch = _between(rng, 1, 64)
        steps = _between(rng, 1, max(1, min(65536, (1 << 25) // (channels * batch))))
        return {"op": op, "batch": batch, "steps": steps, "channels": channels, "group": group, "dtype": dtype,
                "form": rng.choice(["sigmoid", "value"]), "train": rng.random() < 0.6,
                "lengths": rng.random() < 0.4, "resets": rng.random() < 0.4, "state": rng.random() < 0.6}
    cols = _between(rng, 1, 16384)
    rows = _between(rng, 1, max(1, min(65536, (1 << 26) // cols)))
    return {"op": op, "rows": rows, "cols": cols, "pad": rng.choice([0, 0, 0, 1, 8, 47]), "dtype": dtype,
            "p": rng.choice([0.05, 0.1, 0.25, 0.5]), "residual": rng.random() < 0.5, "train": rng.random() < 0.5}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, shift=0.0, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = {"case": case}
    if case["op"] == "dropout":
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        for name in ("x",) + (("r",) if case["residual"] else ()) + (("dy",) if case["train"] else ()):
            s[name] = normal(rows, cols + pad)[:, :cols]
        s["seed"], s["layer"] = (0x5DEECE66D * (seed + 1)) & _M64, seed % 97
        return s
    if case["op"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        x = normal(rows, vocab, scale=2.5)
        # a few tokens stand out, as a trained model's do
        peak = torch.randint(vocab, (rows, 1), generator=g, device="cuda")
        peak = (peak + torch.arange(min(vocab, 4), device="cuda") * max(1, vocab // 4)) % vocab
        x.scatter_(1, peak, normal(rows, peak.shape[1], scale=2.0, shift=9.0))
        if case["masked"]:  # a tenth of the vocabulary is barred
            barred = torch.randperm(vocab, generator=g, device="cuda")[:vocab // 10]
            x[:, barred] = -math.inf
        t = torch.randint(vocab, (rows,), generator=g, device="cuda")
        t = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.5, peak[:, 0], t)
        if case["masked"]:
            t = torch.where(torch.isinf(x.gather(1, t[:, None])[:, 0]), x.argmax(1), t)
        if case["train"] != "no":  # padding of the batch: a token in sixteen has no target
            t = torch.where(torch.rand(rows, generator=g, device="cuda") < 1 / 16, torch.full_like(t, -1), t)
            s["dlp"] = normal(rows, scale=0.2, shift=-1.0, dtype=torch.float32) / rows
            s["dent"] = normal(rows, scale=0.01, dtype=torch.float32) / rows
        s["x"], s["t"] = x, t
        return s
    B, T, D, G = case["batch"], case["steps"], case["channels"], case["channels"] // case["group"]
    s["x"] = normal(B, T, D)
    if case["form"] == "sigmoid":
        s["gate"] = normal(B, T, G, scale=1.5, shift=2.0)
    else:
        s["gate"] = torch.rand((B, T, G), generator=g, device="cuda").mul_(0.3).add_(0.7).to(dt)
    s["h0"] = normal(B, D, dtype=torch.float32) if case["state"] else None
    s["lengths"] = s["reset"] = None
    if case["lengths"]:
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        s["lengths"][-1] = T
    if case["resets"]:
        s["reset"] = torch.rand((B, T), generator=g, device="cuda") < 1 / 512
    if case["train"]:
        s["dy"] = normal(B, T, D)
        s["dh"] = normal(B, D, dtype=torch.float32) if case["state"] else None
    return s


def work(case):
    e = _BYTES[case["dtype"]]
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        tensors = 2 + (1 if case["residual"] else 0) + (2 if case["train"] else 0)
        return {"bytes": n * e * tensors, "flops": n * (2 if case["train"] else 1)}
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        small = case["rows"] * (8 + 12 + 8 * case["top"] + (8 if case["train"] != "no" else 0))
        return {"bytes": n * e * (1 if case["train"] == "no" else 2) + small,
                "flops": n * (5 if case["train"] == "no" else 11)}
    B, T, D, G = case["batch"], case["steps"], case["channels"], case["channels"] // case["group"]
    n, ng = B * T * D, B * T * G
    # x, y, and dy, dx; the gate and its gradient; states
    return {"bytes": e * (n * (4 if case["train"] else 2) + ng * (2 if case["train"] else 1))
            + 4 * B * D * ((2 if case["state"] else 1) + (2 if case["train"] and case["state"] else 0)),
            "flops": n * (20 if case["train"] else 7)}


def run(state):
    return {"dropout": _run_dropout, "logprobs": _run_logprobs, "scan": _run_scan}[state["case"]["op"]](state)


# ---- dropout ---------------------------------------------------------------------------------

_C1, _C2, _C3 = 0x9E3779B97F4A7C15, 0x6A09E667F3BCC909, 0xBB67AE8584CAA73B
_DROPOUT_DOMAIN = 0xA54FF53A5F1D36F1  # keeps these draws apart from those of stochastic rounding


def _signed(v):
    v &= _M64
    return v - (1 << 64) if v >= (1 << 63) else v


def _draws(n, seed, layer, device):
    """32 bits for each of n elements: one 64-bit hash serves elements 2j and 2j + 1."""
    j = torch.arange((n + 1) // 2, device=device, dtype=torch.int64)
    z = j * _signed(_C2) + _signed(seed ^ _DROPOUT_DOMAIN ^ ((layer + 1) * _C1))
    z = z ^ ((z >> 32) & 0xFFFFFFFF)
    z = z * _signed(_C1)
    z = z ^ ((z >> 29) & ((1 << 35) - 1))
    z = z * _signed(_C3)
    high = (z >> 32) & 0xFFFFFFFF
    low = (z ^ high) & 0xFFFFFFFF
    return torch.stack((high, low), 1).reshape(-1)[:n]


def _plain_dropout(x, r, p, seed, layer):
    keep = (_draws(x.numel(), seed, layer, x.device) >= int(round(p * 2.0 ** 32))).reshape(x.shape)
    y = torch.where(keep, x.float() * (1.0 / (1.0 - p)), 0.0)
    if r is not None:
        y = y + r.float()
    return y.to(x.dtype)


def _run_dropout(s):
    p = s["case"]["p"]
    if own:
        from paper_2107_13490_b200 import binding as B
        out = {"y": B.adapt_dropout(s["x"], p, s["seed"], s["layer"], residual=s.get("r"))}
        if "dy" in s:
            out["dx"] = B.adapt_dropout(s["dy"], p, s["seed"], s["layer"])
        return out
    out = {"y": _plain_dropout(s["x"], s.get("r"), p, s["seed"], s["layer"])}
    if "dy" in s:
        out["dx"] = _plain_dropout(s["dy"], None, p, s["seed"], s["layer"])
    return out


def _exact_dropout(s):
    x, p = s["x"], s["case"]["p"]
    n = x.numel()
    with np.errstate(over="ignore"):
        z = np.arange((n + 1) // 2, dtype=np.uint64)
        z *= np.uint64(_C2)
        z += np.uint64((s["seed"] ^ _DROPOUT_DOMAIN ^ ((s["layer"] + 1) * _C1)) & _M64)
        z ^= z >> np.uint64(32)
        z *= np.uint64(_C1)
        z ^= z >> np.uint64(29)
        z *= np.uint64(_C3)
        z ^= z >> np.uint64(32)
    u = z.view(np.uint32).reshape(-1, 2)[:, ::-1].reshape(-1)[:n]  # little-endian: high half first
    keep = torch.from_numpy((u >= np.uint64(round(p * 2.0 ** 32)))).reshape(x.shape).to(x.device)
    scale = lambda v: torch.where(keep, v.double() / (1.0 - p), 0.0)  # noqa: E731
    out = {"y": scale(x) + (s["r"].double() if "r" in s else 0.0)}
    if "dy" in s:
        out["dx"] = scale(s["dy"])
    return out


# ---- token log probabilities -------------------------------------------------------------------

def _top(x, k):
    """The k largest logits of each row, equal ones by the lower index: (ids, logits)."""
    bits = (x.float() + 0.0).view(torch.int32).to(torch.int64)
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
    key = order * (1 << 32) + (0xFFFFFFFF - torch.arange(x.shape[1], device=x.device))
    ids = torch.topk(key, k, dim=1).indices
    return ids.to(torch.int32), x.gather(1, ids).float()


def _plain_logprobs(x, t, scale, k):
    z = x.float() * scale
    m = z.max(1, keepdim=True).values
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    entropy = torch.log(total) - torch.where(e > 0, e * (z - m), 0.0).sum(1, keepdim=True) / total
    live = t >= 0
    logprob = torch.where(live, (z.gather(1, t.clamp(min=0)[:, None]) - lse)[:, 0], 0.0)
    out = {"logprob": logprob, "entropy": torch.where(live, entropy[:, 0], 0.0), "lse": torch.where(live, lse[:, 0], 0.0)}
    if k:
        ids, v = _top(x, k)
        out["top_ids"] = torch.where(live[:, None], ids, -1)
        out["top_logprobs"] = torch.where(live[:, None], v * scale - lse, 0.0)
    return out


def _plain_logprobs_backward(x, t, scale, lse, entropy, dlp, dent):
    live = (t >= 0)[:, None]
    logp = x.float() * scale - lse[:, None]
    p = torch.exp(logp)
    d = -p * dlp[:, None] - dent[:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), 0.0)
    d.scatter_add_(1, t.clamp(min=0)[:, None], dlp[:, None])
    return torch.where(live, d * scale, 0.0).to(x.dtype)


def _run_logprobs(s):
    case, x, t = s["case"], s["x"], s["t"]
    scale, k, train = 1.0 / case["temperature"], case["top"], case["train"]
    if own:
        from paper_2107_13490_b200 import binding as B
        if train == "loss":
            r = B.adapt_token_logprobs(x, t, scale=scale, n_top=k, d_logprob=s["dlp"], d_entropy=s["dent"])
        else:
            r = B.adapt_token_logprobs(x, t, scale=scale, n_top=k)
        out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse}
        if k:
            out["top_ids"], out["top_logprobs"] = r.top_ids, r.top_logprobs
        if train == "loss":
            out["dlogits"] = r.dlogits
        elif train == "later":
            out["dlogits"] = B.adapt_token_logprobs_backward(x, t, r.lse, s["dlp"], r.entropy, s["dent"], scale=scale)
        return out
    out = _plain_logprobs(x, t, scale, k)
    if train != "no":
        out["dlogits"] = _plain_logprobs_backward(x, t, scale, out["lse"], out["entropy"], s["dlp"], s["dent"])
    return out


def _exact_logprobs(s):
    case, t = s["case"], s["t"]
    scale, k = 1.0 / case["temperature"], case["top"]
    rows = s["x"].shape[0]
    parts = []
    step = max(1, (1 << 26) // s["x"].shape[1])
    for i in range(0, rows, step):
        x, ti = s["x"][i:i + step].double(), t[i:i + step]
        dead = ti < 0
        logp = torch.log_softmax(x * scale, 1)
        lse = torch.logsumexp(x * scale, 1)
        p = logp.exp()
        plogp = torch.special.xlogy(p, p)
        h = -plogp.sum(1)
        at = ti.clamp(min=0)[:, None]
        o = {"logprob": logp.gather(1, at)[:, 0], "entropy": h, "lse": lse}
        if k:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
            o["top_ids"], o["top_logprobs"] = ids.to(torch.int32), logp.gather(1, ids)
        if case["train"] != "no":
            dlp, dh = s["dlp"][i:i + step].double()[:, None], s["dent"][i:i + step].double()[:, None]
            hot = torch.zeros_like(p).scatter_(1, at, 1.0)
            o["dlogits"] = scale * (dlp * (hot - p) - dh * (plogp + p * h[:, None]))
        for name, v in o.items():
            v[dead] = -1 if name == "top_ids" else 0
        parts.append(o)
    return {name: torch.cat([o[name] for o in parts]) for name in parts[0]}


# ---- gated linear recurrence ---------------------------------------------------------------------

def _linear_scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 from h_{-1} = 0, by halving the sequence."""
    T = a.shape[1]
    if T == 1:
        return b
    even, odd = slice(0, T - 1, 2), slice(1, T, 2)
    h_odd = _linear_scan(a[:, odd] * a[:, even], a[:, odd] * b[:, even] + b[:, odd])
    h = torch.empty_like(b)
    h[:, odd] = h_odd
    h[:, :1] = b[:, :1]
    inner = slice(2, T, 2)
    h[:, inner] = a[:, inner] * h_odd[:, :(T - 1) // 2] + b[:, inner]
    return h


def _gates(s, x, gate):
    """Coefficients a (of the state) and c (of x), the step's liveness and the kept part of the state."""
    case = s["case"]
    gate = gate.repeat_interleave(case["group"], 2)
    if case["form"] == "sigmoid":
        a, c = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    else:
        a, c = gate, torch.ones_like(gate)
    B, T, _ = x.shape
    live = torch.ones((B, T, 1), dtype=torch.bool, device=x.device)
    if s["lengths"] is not None:
        live = (torch.arange(T, device=x.device)[None] < s["lengths"][:, None])[..., None]
    kept = torch.ones_like(live) if s["reset"] is None else ~s["reset"][..., None]
    return a, c, live, kept


def _plain_scan(s):
    case = s["case"]
    x = s["x"].float()
    a, c, live, kept = _gates(s, x, s["gate"].float())
    dead = ~live
    move = torch.where(dead, 1.0, torch.where(kept, a, 0.0))
    add = torch.where(dead, 0.0, c * x)
    h0 = torch.zeros_like(x[:, 0]) if s["h0"] is None else s["h0"]
    h = _linear_scan(move, torch.cat((add[:, :1] + move[:, :1] * h0[:, None], add[:, 1:]), 1))
    out = {"y": torch.where(live, h, 0.0).to(s["x"].dtype), "h_last": h[:, -1].clone()}
    if not case["train"]:
        return out
    dy = torch.where(live, s["dy"].float(), 0.0)
    if s["dh"] is not None:
        dy[:, -1] += s["dh"]
    back = torch.cat((torch.zeros_like(move[:, :1]), move.flip(1)[:, :-1]), 1)
    dh = _linear_scan(back, dy.flip(1)).flip(1)
    before = torch.where(kept, torch.cat((h0[:, None], h[:, :-1]), 1), 0.0)
    if case["form"] == "sigmoid":
        dgate = dh * (before - x) * a * c
    else:
        dgate = dh * before
    dgate = torch.where(live, dgate, 0.0)
    B, T, D = x.shape
    out["dx"] = torch.where(live, dh * c, 0.0).to(s["x"].dtype)
    out["dgate"] = dgate.reshape(B, T, D // case["group"], case["group"]).sum(3).to(s["x"].dtype)
    if s["h0"] is not None:
        out["dh0"] = move[:, 0] * dh[:, 0]
    return out


def _run_scan(s):
    if not own:
        return _plain_scan(s)
    from paper_2107_13490_b200 import binding as B
    mode = B.GATE_SIGMOID if s["case"]["form"] == "sigmoid" else B.GATE_VALUE
    train = s["case"]["train"]
    r = B.adapt_gated_scan(s["x"], s["gate"], h0=s["h0"], lengths=s["lengths"], reset=s["reset"], mode=mode,
                           want_carry=train)
    out = {"y": r.y, "h_last": r.h_last}
    if train:
        g = B.adapt_gated_scan_backward(s["x"], s["gate"], s["dy"], r.carry, dh_last=s["dh"], lengths=s["lengths"],
                                        reset=s["reset"], mode=mode, want_dh0=s["h0"] is not None)
        out["dx"], out["dgate"] = g.dx, g.dgate
        if s["h0"] is not None:
            out["dh0"] = g.dh0
    return out


def _exact_scan(s):
    case = s["case"]
    x = s["x"].double()
    B, T, D = x.shape
    if B * T * D > 1 << 27:
        return None
    gate = s["gate"].double().repeat_interleave(case["group"], 2)
    a = torch.sigmoid(gate) if case["form"] == "sigmoid" else gate
    c = torch.sigmoid(-gate) if case["form"] == "sigmoid" else torch.ones_like(gate)
    move, add = a.clone(), c * x
    if s["reset"] is not None:
        move[s["reset"]] = 0.0
    live = None
    if s["lengths"] is not None:
        live = torch.arange(T, device=x.device)[None, :, None] < s["lengths"][:, None, None]
        move = move.masked_fill(~live, 1.0)
        add = add.masked_fill(~live, 0.0)
    h = torch.zeros((B, D), dtype=torch.float64, device=x.device) if s["h0"] is None else s["h0"].double()
    before = torch.empty_like(x)
    y = torch.empty_like(x)
    for t in range(T):
        before[:, t] = h
        h = torch.addcmul(add[:, t], move[:, t], h)
        y[:, t] = h
    only = (lambda v: v) if live is None else (lambda v: v.masked_fill(~live, 0.0))
    out = {"y": only(y), "h_last": h}
    if not case["train"]:
        return out
    dy = only(s["dy"].double())
    flow = torch.zeros((B, D), dtype=torch.float64, device=x.device) if s["dh"] is None else s["dh"].double()
    dh = torch.empty_like(x)
    for t in reversed(range(T)):
        torch.add(dy[:, t], flow, out=dh[:, t])
        flow = move[:, t] * dh[:, t]
    if s["reset"] is not None:
        before[s["reset"]] = 0.0
    dg = dh * (before - x) * a * c if case["form"] == "sigmoid" else dh * before
    out["dx"] = only(dh * c)
    out["dgate"] = only(dg).reshape(B, T, D // case["group"], case["group"]).sum(3)
    if s["h0"] is not None:
        out["dh0"] = flow
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"dropout": _exact_dropout, "logprobs": _exact_logprobs, "scan": _exact_scan}[case["op"]](s)
