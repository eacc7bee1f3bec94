"""The operators around the layers together, as the example's model with norms uses them: its gradients, its single-token
form, and its products on 8-bit codes."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def LM():
    import torch
    assert torch.cuda.is_available()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent_lm.py")
    spec = importlib.util.spec_from_file_location("recurrent_lm", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def model_of(LM, vocab, width, layers):
    import torch
    model = LM.RecurrentLM(vocab, width, layers, dtype=torch.float32, norms=True)
    gen = torch.Generator(device="cuda").manual_seed(6)
    model.used = [w + 0.1 * torch.randn(w.shape, generator=gen, device="cuda") if w.dim() == 1 else w for w in model.used]
    return model


@pytest.mark.parametrize("width", [16, 33])
def test_gradients_against_differences_of_the_loss(LM, width):
    import torch
    model = model_of(LM, 50, width, 2)
    tokens, targets, reset = LM.synthetic_text(3, 70, 50, 1)
    loss, gradients = model.loss_and_gradients(tokens, targets, reset, p=0.25, seed=9)
    assert len(gradients) == len(model.names) == 2 + 3 * 2 + 5
    gen = torch.Generator(device="cuda").manual_seed(0)
    base = model.used
    direction = [torch.randn(w.shape, generator=gen, device="cuda") * 0.1 for w in base]
    want = sum((g.double() * d.double()).sum() for g, d in zip(gradients, direction))
    slopes = []
    for eps in (2.0 ** -6, 2.0 ** -7):
        value = []
        for s in (eps, -eps):
            model.used = [w + s * d for w, d in zip(base, direction)]
            value.append(model.loss_and_gradients(tokens, targets, reset, p=0.25, seed=9)[0].double())
        slopes.append((value[0] - value[1]) / (2 * eps))
    # central differences at h and h / 2: the error in h^2 is a third of their own difference at the smaller step, what
    # follows it (h^4) less; the loss (about 4, in fp32 through some ten roundings a layer) is good to 2^-20
    tol = abs(slopes[0] - slopes[1]) + 8 * 2.0 ** -20 / 2.0 ** -7
    assert abs(slopes[1] - want) <= tol, (slopes, float(want), float(tol))


def test_single_tokens_give_the_sequence_s_logits(LM):
    import torch
    model = model_of(LM, 40, 32, 2)
    tokens = torch.randint(40, (3, 20), device="cuda")
    reset = torch.zeros((3, 20), dtype=torch.bool, device="cuda")
    whole = model.logits(model.used, tokens, reset, 0.0, 0).reshape(3, 20, 40)
    state = model.step_state(3)
    for t in range(20):
        r = model.next_tokens(tokens[:, t], state, n_top=1)
    lse = torch.logsumexp(whole[:, -1].double(), 1)
    assert torch.allclose(r.lse.double(), lse, rtol=1e-5, atol=1e-5)
    assert LM.continue_text(model, tokens[:, :4], 5, int8=True).shape == (3, 5)


def test_products_on_codes(LM):
    """One step on codes against the same step with each product's operands replaced by what their codes stand for."""
    import torch
    B = LM.B
    model = model_of(LM, 64, 48, 2)
    codes = model.codes()
    w = dict(zip(model.names, model.used))
    tokens = torch.randint(64, (5,), device="cuda")
    state, want_state = model.step_state(5), model.step_state(5)

    def product(x, name):
        x, c = B.adapt_int8_rows(x.contiguous()), codes[name]
        return ((x.codes.double() * x.scales.double()[:, None]) @ (c.codes.double() * c.scales.double()[:, None]).t()).float()

    for _ in range(3):
        got = model.next_tokens(tokens, state, n_top=3, codes=codes)
        x = w["embed"][tokens]
        n = B.adapt_block_norm(x, weight_before=w["before0"], want_y=False).normed
        for i in range(2):
            u, gate = product(n, f"in{i}"), product(n, f"gate{i}")
            h = B.adapt_gated_scan(u[:, None], gate[:, None] + 1, h0=want_state[i], h_last=want_state[i]).y[:, 0]
            r = B.adapt_block_norm(product(h, f"out{i}"), residual=x, weight_after=w[f"after{i}"], weight_before=w[f"before{i + 1}"], after=B.NORM_RMS)
            x, n = r.y, r.normed
        # a rounding of an activation next to the border of two codes may fall either way: one of 48 products by 1 / 127
        # of the largest activation and a weight
        want = B.adapt_token_logprobs(product(n, "head"))
        assert (got.lse - want.lse).abs().max() <= 0.02


def test_runs_with_the_precision_switch(LM):
    model, losses, formats = LM.train(steps=12, batch=4, length=32, width=64, vocab=96, layers=2, every=5, norms=True, say=None)
    assert losses.isfinite().all() and formats.shape[0] == len(model.names)


def test_a_captured_step_replays(LM):
    """Embedding, norms and products of one decoding step in a CUDA graph, replayed on other tokens."""
    import torch
    model = model_of(LM, 64, 64, 2)
    codes, state = model.codes(), model.step_state(4)
    tokens = torch.randint(64, (4,), device="cuda")
    model.next_tokens(tokens, state, codes=codes)
    graph, held = torch.cuda.CUDAGraph(), model.step_state(4)
    with torch.cuda.graph(graph):
        out = model.next_tokens(tokens, held, codes=codes)
    for _ in range(3):
        tokens.copy_(torch.randint(64, (4,), device="cuda"))
        for h in held + state:
            h.zero_()
        graph.replay()
        want = model.next_tokens(tokens, state, codes=codes)
        assert torch.equal(out.lse, want.lse) and torch.equal(out.top_ids, want.top_ids)
