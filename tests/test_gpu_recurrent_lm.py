"""The training-step operators together: the example's model, its gradients and its single-token form."""
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


def test_training_lowers_the_loss(LM):
    model, losses, formats = LM.train(steps=30, batch=8, length=64, width=64, vocab=128, layers=2, say=None)
    assert losses.isfinite().all()
    assert float(losses[-5:].mean()) < 0.8 * float(losses[:5].mean())
    assert (formats[:, 0] >= 4).all() and (formats[:, 0] <= 32).all()
    for used, w, (wl, fl) in zip(model.used, model.weights, formats[:, :2].tolist()):
        code = used * 2.0 ** fl                   # the weights in use are fixed-point numbers
        assert (code == code.round()).all() and (code.abs() <= 2.0 ** (wl - 1)).all()


def test_gradients_against_differences_of_the_loss(LM):
    import torch
    model = LM.RecurrentLM(50, 16, 2, dtype=torch.float32)
    tokens, targets, reset = LM.synthetic_text(3, 70, 50, 1)
    loss, gradients = model.loss_and_gradients(tokens, targets, reset, p=0.25, seed=9)
    gen = torch.Generator(device="cuda").manual_seed(0)
    direction = [torch.randn(w.shape, generator=gen, device="cuda") * 0.25 for w in model.weights]
    want = sum((g.double() * d.double()).sum() for g, d in zip(gradients, direction))
    eps = 2.0 ** -8
    value = []
    for s in (eps, -eps):
        model.used = [w + s * d for w, d in zip(model.weights, direction)]
        value.append(model.loss_and_gradients(tokens, targets, reset, p=0.25, seed=9)[0].double())
    difference = (value[0] - value[1]) / (2 * eps)
    # the loss (about 4) is good to 2^-20; the third derivative along the direction is of order 100
    tol = 4 * 2.0 ** -20 / eps + 100 * eps ** 2
    assert abs(difference - want) <= tol, (float(difference), float(want), tol)


def test_single_tokens_give_the_sequence_s_logits(LM):
    import torch
    model = LM.RecurrentLM(40, 32, 2, dtype=torch.float32)
    tokens = torch.randint(40, (3, 20), device="cuda")
    reset = torch.zeros((3, 20), dtype=torch.bool, device="cuda")
    whole = model.logits(model.used, tokens, reset, 0.0, 0).reshape(3, 20, 40)
    state = model.step_state(3)
    for t in range(20):
        r = model.next_tokens(tokens[:, t], state, n_top=1)
    lse = torch.logsumexp(whole[:, -1].double(), 1)
    assert torch.allclose(r.lse.double(), lse, rtol=1e-5, atol=1e-5)
    assert LM.continue_text(model, tokens[:, :4], 5).shape == (3, 5)


def test_a_batch_without_targets_has_no_loss(LM):
    import torch
    model = LM.RecurrentLM(30, 16, 1, dtype=torch.float32)
    tokens, targets, reset = LM.synthetic_text(2, 20, 30, 3)
    loss, gradients = model.loss_and_gradients(tokens, torch.full_like(targets, -1), reset)
    assert float(loss) == 0 and all((g == 0).all() for g in gradients)
