"""The training-step operators' calls from torch tensors: what they refuse, and how."""
import pytest
import torch

from paper_2107_13490_b200 import binding as B
from paper_2107_13490_b200 import build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_extension_is_required(monkeypatch):
    monkeypatch.setattr(B, "_calls", None)
    monkeypatch.setattr(B, "CALLS_PATH", "/nonexistent/_adapt_torch.so")
    with pytest.raises(RuntimeError, match="build it"):
        B.adapt_dropout(torch.zeros(4), 0.5)


def test_host_tensors_and_other_objects_are_refused():
    x, m = torch.zeros(2, 3, 4), torch.zeros(3, 4)
    for call in (lambda: B.adapt_dropout(x, 0.5), lambda: B.adapt_token_logprobs(m),
                 lambda: B.adapt_token_logprobs_backward(m, None, m[:, 0]), lambda: B.adapt_gated_scan(x, x),
                 lambda: B.adapt_gated_scan_backward(x, x, x, x), lambda: B.adapt_dropout([1.0], 0.5),
                 lambda: B.adapt_token_logprobs(None)):
        with pytest.raises(AssertionError):
            call()


@pytest.mark.gpu
def test_arguments_that_do_not_fit_are_refused():
    x = torch.zeros(6, 40, device="cuda")
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    d = torch.zeros(6, device="cuda")
    s, g = torch.zeros(2, 5, 64, device="cuda"), torch.zeros(2, 5, 16, device="cuda")
    h = torch.zeros(2, 64, device="cuda")
    carry = B.adapt_gated_scan(s, g, want_carry=True).carry
    back = lambda **k: B.adapt_gated_scan_backward(s, g, **{"dy": s, "carry": carry, **k})  # noqa: E731
    for call in (
            lambda: B.adapt_dropout(x.double(), 0.5),
            lambda: B.adapt_dropout(x, 0.5, residual=x[:5]),
            lambda: B.adapt_dropout(x, 0.5, residual=x.half()),
            lambda: B.adapt_dropout(x, 0.5, out=x.cpu()),
            lambda: B.adapt_dropout(x.t(), 0.5),
            lambda: B.adapt_dropout(s.transpose(1, 2), 0.5),
            lambda: B.adapt_token_logprobs(x, t[:5]),
            lambda: B.adapt_token_logprobs(x, t.int()),
            lambda: B.adapt_token_logprobs(x, t.cpu()),
            lambda: B.adapt_token_logprobs(x, t, n_top=33),
            lambda: B.adapt_token_logprobs(x, t, n_top=-1),
            lambda: B.adapt_token_logprobs(x[0], t),
            lambda: B.adapt_token_logprobs(x.t(), t),
            lambda: B.adapt_token_logprobs(x, t, d_logprob=d.double()),
            lambda: B.adapt_token_logprobs(x, t, d_logprob=d, dlogits=x.half()),
            lambda: B.adapt_token_logprobs_backward(x, t, d[:3], d),
            lambda: B.adapt_token_logprobs_backward(x, t, d, d, out=x[:3]),
            lambda: B.adapt_gated_scan(s, g[:1]),
            lambda: B.adapt_gated_scan(s, g[..., :15]),
            lambda: B.adapt_gated_scan(s, g.half()),
            lambda: B.adapt_gated_scan(s, g, h0=h[:, :63]),
            lambda: B.adapt_gated_scan(s, g, h0=h.double()),
            lambda: B.adapt_gated_scan(s, g, h_last=h.t()),
            lambda: B.adapt_gated_scan(s, g, lengths=t[:2]),
            lambda: B.adapt_gated_scan(s, g, reset=d),
            lambda: B.adapt_gated_scan(s.transpose(1, 2).contiguous().transpose(1, 2), g),
            lambda: back(dy=g), lambda: back(carry=carry[:, :0]), lambda: back(dh_last=h[:1]),
            lambda: back(dx=g), lambda: back(dgate=s)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: B.adapt_dropout(x, 1.5), lambda: B.adapt_token_logprobs(x, t, scale=-1.0),
                 lambda: B.adapt_token_logprobs(x[:, :3], t, n_top=4), lambda: B.adapt_token_logprobs(x, t, dlogits=x),
                 lambda: B.adapt_token_logprobs(x, None, d_logprob=d), lambda: B.adapt_token_logprobs_backward(x, t, d),
                 lambda: B.adapt_gated_scan(s, g, mode=7)):
        with pytest.raises(B.AdaptError) as e:
            call()
        assert e.value.status == B.ERR_INVALID_ARG
    for call in (lambda: B.adapt_dropout(x, "half"), lambda: B.adapt_dropout(x, 0.5, seed=1.5),
                 lambda: B.adapt_token_logprobs(x, t, n_top="3")):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_outputs_that_are_not_asked_for_are_none():
    x = torch.randn(3, 50, device="cuda")
    r = B.adapt_token_logprobs(x)
    assert r.logprob is None and r.top_ids is None and r.top_logprobs is None and r.dlogits is None
    assert r.entropy.shape == r.lse.shape == (3,)
    assert B.adapt_token_logprobs(x, want_entropy=False).entropy is None
    s = torch.randn(1, 4, 8, device="cuda")
    r = B.adapt_gated_scan(s, s)
    assert r.carry is None and r.h_last.shape == (1, 8)
    # a sequence of no steps hands the state through
    h = torch.randn(1, 8, device="cuda")
    assert torch.equal(B.adapt_gated_scan(s[:, :0], s[:, :0], h0=h).h_last, h)
    assert B.adapt_dropout(x[:0], 0.5).shape == (0, 50) and B.adapt_token_logprobs(x[:0]).lse.shape == (0,)
    # seeds and layers beyond 32 bits and negative ones are taken modulo their width
    assert torch.equal(B.adapt_dropout(x, 0.5, seed=-1), B.adapt_dropout(x, 0.5, seed=2 ** 64 - 1))


@pytest.mark.gpu
def test_side_tensors_of_another_device_are_refused(monkeypatch):
    """Targets, weights, lengths, resets and states that lie on another GPU.  (Fake tensors: they carry a device,
    and no memory that a kernel could reach.)"""
    from torch._subclasses import fake_tensor
    monkeypatch.setattr(fake_tensor, "init_gpu_context", lambda device: None)   # (it would allocate on that device)

    def away(*shape, dtype=torch.float32):
        with fake_tensor.FakeTensorMode():
            return torch.empty(shape, dtype=dtype, device="cuda:1")

    x = torch.zeros(6, 40, device="cuda")
    t, d = torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros(6, device="cuda")
    s, g, h = torch.zeros(2, 5, 64, device="cuda"), torch.zeros(2, 5, 16, device="cuda"), away(2, 64)
    carry = B.adapt_gated_scan(s, g, want_carry=True).carry
    ft, fd = away(6, dtype=torch.int64), away(6)
    assert ft.device == torch.device("cuda:1") and ft.is_cuda
    back = lambda **k: B.adapt_gated_scan_backward(s, g, **{"dy": s, "carry": carry, **k})  # noqa: E731
    before = B.adapt_kernel_launch_count()
    for call in (lambda: B.adapt_token_logprobs(x, ft), lambda: B.adapt_token_logprobs(x, t, d_logprob=fd),
                 lambda: B.adapt_token_logprobs(x, t, d_entropy=fd),
                 lambda: B.adapt_token_logprobs_backward(x, ft, d, d), lambda: B.adapt_token_logprobs_backward(x, t, fd, d),
                 lambda: B.adapt_token_logprobs_backward(x, t, d, fd),
                 lambda: B.adapt_token_logprobs_backward(x, t, d, d, fd, d),
                 lambda: B.adapt_token_logprobs_backward(x, t, d, d, d, fd),
                 lambda: B.adapt_gated_scan(s, g, h0=h), lambda: B.adapt_gated_scan(s, g, h_last=h),
                 lambda: B.adapt_gated_scan(s, g, lengths=away(2, dtype=torch.int32)),
                 lambda: B.adapt_gated_scan(s, g, reset=away(2, 5, dtype=torch.uint8)),
                 lambda: back(dh_last=h), lambda: back(carry=away(*carry.shape)),
                 lambda: back(lengths=away(2, dtype=torch.int32)), lambda: back(reset=away(2, 5, dtype=torch.bool))):
        with pytest.raises(AssertionError):
            call()
    assert B.adapt_kernel_launch_count() == before


@pytest.mark.gpu
def test_batches_of_no_rows():
    x, t, d = (torch.zeros(0, 40, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"),
               torch.zeros(0, device="cuda"))
    r = B.adapt_token_logprobs(x, t, n_top=4, d_logprob=d, d_entropy=d)
    assert r.top_ids.shape == r.top_logprobs.shape == (0, 4) and r.dlogits.shape == (0, 40)
    assert r.logprob.shape == r.entropy.shape == r.lse.shape == (0,)
    assert B.adapt_token_logprobs_backward(x, t, r.lse, d, r.entropy, d).shape == (0, 40)


@pytest.mark.gpu
def test_numbers_are_taken_as_they_stand():
    x = torch.randn(3, 50, device="cuda")
    s = torch.randn(2, 5, 64, device="cuda")
    carry = B.adapt_gated_scan(s, s, want_carry=True).carry
    for call in (lambda: B.adapt_token_logprobs(x, n_top=2 ** 32 + 1), lambda: B.adapt_token_logprobs(x, n_top=2 ** 64),
                 lambda: B.adapt_token_logprobs(x, n_top=-2 ** 70), lambda: B.adapt_gated_scan(s, s, mode=2 ** 32),
                 lambda: B.adapt_gated_scan_backward(s, s, s, carry, mode=2 ** 32 + 1)):
        with pytest.raises(AssertionError):
            call()
    # a flag without a truth value is an error of its own kind
    many = torch.zeros(2)
    for call in (lambda: B.adapt_token_logprobs(x, want_entropy=many), lambda: B.adapt_gated_scan(s, s, want_carry=many),
                 lambda: B.adapt_gated_scan_backward(s, s, s, carry, want_dh0=many)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            call()
