"""A small recurrent language model trained the AdaPT way, on synthetic text.

Every layer's weights are held in fp32 and used at the fixed-point format that the precision switch
chose for them.  A step runs embedding -> [gated recurrence -> projection -> dropout + residual] x
layers -> vocabulary projection -> loss; its gradients are normalised (adapt_normalize_gradients),
kept for the gradient diversity, and every few steps PushDown (the search) and PushUp choose the next
formats.  Afterwards the model continues a text one token at a time: the recurrence's single-step form
with its state, and the token log probabilities' alternatives.

    python examples/recurrent_lm.py [--steps 60] [--batch 16] [--length 128] [--width 128] [--vocab 512]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2107_13490_b200 import binding as B  # noqa: E402
from paper_2107_13490_b200 import workloads as W  # noqa: E402


class GatedScan(torch.autograd.Function):
    """y = adapt_gated_scan(x, gate) with resets at document starts."""

    @staticmethod
    def forward(ctx, x, gate, reset):
        r = B.adapt_gated_scan(x, gate, reset=reset, want_carry=True)
        ctx.save_for_backward(x, gate, reset, r.carry)
        return r.y

    @staticmethod
    def backward(ctx, dy):
        x, gate, reset, carry = ctx.saved_tensors
        g = B.adapt_gated_scan_backward(x, gate, dy.contiguous(), carry, reset=reset)
        return g.dx, g.dgate, None


class DropoutAdd(torch.autograd.Function):
    """residual + dropout(x); the backward pass draws the same mask again."""

    @staticmethod
    def forward(ctx, x, residual, p, seed, layer):
        ctx.key = (p, seed, layer)
        return B.adapt_dropout(x, p, seed, layer, residual=residual)

    @staticmethod
    def backward(ctx, dy):
        dy = dy.contiguous()
        return B.adapt_dropout(dy, *ctx.key), dy, None, None, None


class TokenLoss(torch.autograd.Function):
    """Mean negative log probability of the targets (negative ones are left out; without any it is 0); the gradient
    comes out of the forward call."""

    @staticmethod
    def forward(ctx, logits, targets):
        live = targets >= 0
        weight = -live.float() / live.sum().clamp(min=1)
        r = B.adapt_token_logprobs(logits, targets, want_entropy=False, d_logprob=weight)
        ctx.save_for_backward(r.dlogits)
        return (r.logprob * weight).sum()

    @staticmethod
    def backward(ctx, d):
        (dlogits,) = ctx.saved_tensors
        return dlogits * d, None


class RecurrentLM:
    """Weights in fp32; `used` are their values at the chosen fixed-point formats."""

    def __init__(self, vocab: int, width: int, layers: int, seed: int = 0, dtype=torch.bfloat16):
        g = torch.Generator().manual_seed(seed)
        scale = width ** -0.5
        make = lambda *s: (torch.randn(s, generator=g) * scale).cuda()  # noqa: E731
        self.names, self.weights, self.layers, self.dtype = [], [], layers, dtype
        for name, shape in [("embed", (vocab, width))] + \
                [(f"{k}{i}", (width, width)) for i in range(layers) for k in ("in", "gate", "out")] + \
                [("head", (width, vocab))]:
            self.names.append(name)
            self.weights.append(make(*shape))
        self.used = [w.clone() for w in self.weights]

    def logits(self, weights, tokens, reset, p, seed):
        w = dict(zip(self.names, weights))
        x = w["embed"].to(self.dtype)[tokens]
        for i in range(self.layers):
            u, gate = (x @ w[f"{k}{i}"].to(self.dtype) for k in ("in", "gate"))
            h = GatedScan.apply(u, gate + 1, reset)     # + 1: states begin as long memories
            x = DropoutAdd.apply(h @ w[f"out{i}"].to(self.dtype), x, p, seed, i)
        return x.reshape(-1, x.shape[-1]) @ w["head"].to(self.dtype)

    def loss_and_gradients(self, tokens, targets, reset, p=0.1, seed=0):
        """One forward and backward pass at the used (fixed-point) weights."""
        weights = [w.detach().requires_grad_() for w in self.used]
        loss = TokenLoss.apply(self.logits(weights, tokens, reset, p, seed), targets.reshape(-1))
        return loss.detach(), [g.contiguous() for g in torch.autograd.grad(loss, weights)]

    def step_state(self, batch: int):
        width = self.weights[0].shape[1]
        return [torch.zeros((batch, width), device="cuda") for _ in range(self.layers)]

    def next_tokens(self, tokens, state, n_top=4):
        """One token for every sequence: alternatives of the next; the states move on in place."""
        w = dict(zip(self.names, self.used))
        x = w["embed"].to(self.dtype)[tokens][:, None]
        for i in range(self.layers):
            u, gate = (x @ w[f"{k}{i}"].to(self.dtype) for k in ("in", "gate"))
            h = B.adapt_gated_scan(u, gate + 1, h0=state[i], h_last=state[i]).y
            x = x + h @ w[f"out{i}"].to(self.dtype)
        return B.adapt_token_logprobs(x[:, 0] @ w["head"].to(self.dtype), n_top=n_top)


def synthetic_text(batch: int, length: int, vocab: int, step: int):
    """Documents of random length in which every token follows from the one before it, but for one in
    eight that is random: (tokens, targets, reset)."""
    g = torch.Generator().manual_seed(step)
    t = torch.randint(vocab, (batch, length + 1), generator=g)
    noise = torch.rand((batch, length + 1), generator=g) < 0.125
    reset = torch.rand((batch, length), generator=g) < 1 / 64
    reset[:, 0] = True
    for i in range(1, length + 1):
        follows = (5 * t[:, i - 1] + 17) % vocab
        begins = reset[:, i] if i < length else torch.zeros(batch, dtype=torch.bool)
        t[:, i] = torch.where(noise[:, i] | begins, t[:, i], follows)
    targets = t[:, 1:].clone()
    targets[:, :-1][reset[:, 1:]] = -1      # nothing foretells a document's first token
    return t[:, :-1].cuda(), targets.cuda(), reset.cuda()


class PrecisionSwitch:
    """PushDown and PushUp over the weights and the last gradients (lookback)."""

    def __init__(self, model: RecurrentLM, lookback: int = 5, buff: int = 4, n_bins: int = 100, eps: float = 1e-3):
        self.model, self.lookback, self.buff, self.n_bins, self.eps = model, lookback, buff, n_bins, eps
        self.grid = B.Grid(*W.candidate_grid(range(4, 25)))
        self.history = [[] for _ in model.weights]
        self.formats = None

    def keep(self, gradients):
        for kept, g in zip(self.history, gradients):
            kept.append(g)
            del kept[:-self.lookback]

    def switch(self):
        best = B.adapt_precision_search_ex(self.model.weights, self.grid, self.n_bins, eps=self.eps).best
        diversity = B.adapt_gradient_diversity(self.history)
        pushed = B.adapt_pushup(diversity, best, B.STRATEGY_MEAN, self.buff)
        formats = best.cpu()
        formats[:, :2] = torch.from_numpy(pushed)
        self.formats = formats.cuda()

    def apply(self):
        if self.formats is not None:
            B.adapt_requantize_selected_batch(self.model.weights, self.formats, values_out=self.model.used)
        else:
            for u, w in zip(self.model.used, self.model.weights):
                u.copy_(w)


def train(steps=60, batch=16, length=128, width=128, vocab=512, layers=2, rate=0.3, every=10, p=0.1, say=print):
    """Trains and returns (model, losses, formats)."""
    model = RecurrentLM(vocab, width, layers)
    switch = PrecisionSwitch(model)
    losses = []
    for step in range(steps):
        switch.apply()
        tokens, targets, reset = synthetic_text(batch, length, vocab, step)
        loss, gradients = model.loss_and_gradients(tokens, targets, reset, p=p, seed=step)
        losses.append(loss)
        switch.keep(gradients)
        scale = rate * (1 - step / steps)
        for w, g in zip(model.weights, B.adapt_normalize_gradients(gradients)):
            w.sub_(g, alpha=scale)
        if step % every == every - 1:
            switch.switch()
            if say:
                wl = switch.formats[:, :2].tolist()
                say(f"step {step + 1}: loss {float(loss):.3f}, <WL,FL> " +
                    " ".join(f"{n}<{a},{b}>" for n, (a, b) in zip(model.names, wl)))
    switch.apply()
    return model, torch.stack(losses).cpu(), switch.formats


def continue_text(model: RecurrentLM, prompt, n: int):
    """Greedy continuation, token by token."""
    state = model.step_state(prompt.shape[0])
    for t in prompt.unbind(1):
        r = model.next_tokens(t, state)
    out = []
    for _ in range(n):
        out.append(r.top_ids[:, 0].long())
        r = model.next_tokens(out[-1], state)
    return torch.stack(out, 1)


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("steps", 60), ("batch", 16), ("length", 128), ("width", 128), ("vocab", 512), ("layers", 2)):
        a.add_argument(f"--{name}", type=int, default=value)
    o = vars(a.parse_args())
    model, losses, _ = train(**o)
    prompt = torch.randint(o["vocab"], (2, 1), device="cuda")
    print("loss", f"{float(losses[:5].mean()):.3f} -> {float(losses[-5:].mean()):.3f}")
    print("prompt", prompt[:, 0].tolist(), "continued by", continue_text(model, prompt, 8).tolist())


if __name__ == "__main__":
    main()
