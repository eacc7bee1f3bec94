"""The gated recurrence against the 64-bit reference.

Bounds (fp32 arithmetic): a step's a, c x and their combination carry a relative error of at most
d = 2^-20 (exponential, reciprocal and a few roundings, or the roundings of a product of decays), so the
state's error obeys E_t = |a_t| E_{t-1} + d H_t with H_t = |a_t| H_{t-1} + |c_t x_t| - the same
recurrence on magnitudes - and the gradient's likewise in reverse.  Outputs are rounded once to their type."""
import math

import numpy as np
import pytest

from tests import training_reference as R

pytestmark = pytest.mark.gpu

D_STEP = 2.0 ** -20
UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -126, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -126}
DTYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2107_13490_b200 import binding
    binding.lib()
    return binding


def flip(v, lengths, T):
    """Each sequence's first n steps in reverse."""
    out = np.zeros_like(v)
    for b in range(v.shape[0]):
        n = T if lengths is None else max(0, min(T, int(lengths[b])))
        out[b, :n] = v[b, :n][::-1]
    return out


def shift_gate(a, reset):
    """Decays as the reversed pass meets them: the decay of step t + 1 moves the gradient to t."""
    out = a.copy()
    if reset is not None:
        out[reset != 0] = 0
    return out


def reference(x, gate, h0, lengths, reset, sigmoid, dy=None, dl=None):
    """Values and bounds: {name: (value, absolute bound without the output's rounding)}."""
    B, T, D = x.shape
    group = D // gate.shape[2]
    g = np.repeat(gate, group, 2)
    with np.errstate(over="ignore"):
        a = 1 / (1 + np.exp(-g)) if sigmoid else g
        c = 1 / (1 + np.exp(g)) if sigmoid else np.ones_like(g)
    ax, zero = np.abs(c * x), np.zeros((B, D))
    size = R.scan(ax, np.abs(a), None if h0 is None else np.abs(h0), lengths, reset, False)
    err = R.scan(D_STEP * size[0], np.abs(a), zero, lengths, reset, False)
    if dy is None:
        y, h, _ = R.scan(x, gate, h0, lengths, reset, sigmoid)
        return {"y": (y, err[0]), "h_last": (h, err[1])}
    (y, h, before), (dx, dg, dh0) = R.scan(x, gate, h0, lengths, reset, sigmoid, dy, dl)
    # the gradient flow on magnitudes, and its error, by the formula's own reference
    keep = np.abs(shift_gate(a, reset))
    (_, _, _), (mag, _, flow) = R.scan(ax, keep, None, lengths, None, False, np.abs(dy), None if dl is None else np.abs(dl))
    (_, _, _), (merr, _, flow_err) = R.scan(ax, keep, None, lengths, None, False, D_STEP * (mag + np.abs(dy)), zero)
    e_before, s_before = err[2], size[2]
    ax_raw = np.abs(x) if sigmoid else 0
    slope = np.abs(a * c) if sigmoid else 1.0
    dx_tol = np.abs(c) * (merr + D_STEP * mag)
    dg_tol = slope * (merr * (s_before + ax_raw) + mag * (e_before + D_STEP * (s_before + ax_raw)))
    terms = slope * mag * (s_before + ax_raw)
    dg_tol = (dg_tol + (group + 1) * 2.0 ** -24 * terms).reshape(B, T, D // group, group).sum(3)
    return {"y": (y, err[0]), "h_last": (h, err[1]), "dx": (dx, dx_tol), "dgate": (dg, dg_tol),
            "dh0": (dh0, flow_err + D_STEP * flow)}


def close(name, got, want, dtype):
    value, tol = want
    if name in ("h_last", "dh0"):
        dtype = "float32"
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isfinite(got), np.isfinite(value)), name
    fine = np.isfinite(value)
    err = np.abs(got - value)[fine]
    bound = (tol + UNIT[dtype] * np.abs(value) * 1.01 + TINY[dtype])[fine]
    assert (err <= bound).all(), (name, float((err / bound).max()))


def arr(t):
    return None if t is None else t.double().cpu().numpy()


def case(dtype, batch, steps, channels, group, seed, sigmoid, state=True, lengths=None, resets=False):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, dtype)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    c = {"x": rand(batch, steps, channels).to(dt), "dy": rand(batch, steps, channels).to(dt)}
    G = channels // group
    c["gate"] = ((rand(batch, steps, G) * 2 + 1) if sigmoid else torch.tanh(rand(batch, steps, G)) * 1.02).to(dt)
    c["h0"] = rand(batch, channels) if state else None
    c["dl"] = rand(batch, channels) if state else None
    c["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    c["reset"] = (torch.rand((batch, steps), generator=g, device="cuda") < 0.05) if resets else None
    return c


def run(B, c, sigmoid, **k):
    mode = B.GATE_SIGMOID if sigmoid else B.GATE_VALUE
    r = B.adapt_gated_scan(c["x"], c["gate"], h0=c["h0"], lengths=c["lengths"], reset=c["reset"], mode=mode,
                           want_carry=True, **k)
    g = B.adapt_gated_scan_backward(c["x"], c["gate"], c["dy"], r.carry, dh_last=c["dl"], lengths=c["lengths"],
                                    reset=c["reset"], mode=mode, want_dh0=True)
    return {"y": r.y, "h_last": r.h_last, "dx": g.dx, "dgate": g.dgate, "dh0": g.dh0}


def check(B, c, sigmoid):
    dtype = str(c["x"].dtype).split(".")[1]
    got = run(B, c, sigmoid)
    reset = None if c["reset"] is None else c["reset"].cpu().numpy().astype(np.uint8)
    lengths = None if c["lengths"] is None else c["lengths"].cpu().numpy()
    want = reference(arr(c["x"]), arr(c["gate"]), arr(c["h0"]), lengths, reset, sigmoid, arr(c["dy"]), arr(c["dl"]))
    for name in want:
        close(name, got[name], want[name], dtype)
    return got


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("batch,steps,channels", [(1, 1, 1), (3, 1, 70), (2, 2, 64), (1, 5, 33), (2, 15, 65), (2, 16, 128),
                                                  (1, 17, 2), (3, 127, 66), (2, 128, 64), (2, 129, 130), (1, 300, 96),
                                                  (2, 1000, 10)])
def test_sizes(B, sigmoid, dtype, batch, steps, channels):
    check(B, case(dtype, batch, steps, channels, 1, steps + channels, sigmoid), sigmoid)


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_long_sequences(B, sigmoid, dtype):
    check(B, case(dtype, 1, 5003, 72, 1, 7, sigmoid), sigmoid)
    check(B, case(dtype, 3, 4111, 2, 1, 7, sigmoid, resets=True), sigmoid)


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group,channels", [(2, 64), (2, 66), (4, 12), (8, 200), (16, 48), (32, 96), (64, 64), (64, 192),
                                            (128, 256), (192, 192), (256, 256)])
def test_shared_gates(B, sigmoid, dtype, group, channels):
    for steps in (3, 131):
        check(B, case(dtype, 2, steps, channels, group, group, sigmoid, resets=True), sigmoid)


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
def test_lengths_and_resets(B, sigmoid, dtype):
    for steps in (4, 140, 400):
        for resets in (False, True):
            lengths = [0, 1, steps, steps - 1, steps // 2, 128, -3, steps + 9]
            c = case(dtype, len(lengths), steps, 40, 1, steps, sigmoid, lengths=lengths, resets=resets)
            if resets:
                c["reset"][2, 0] = c["reset"][3, -2] = True
                c["reset"][:, min(128, steps - 1)] = True     # at a tile's first step
            got = check(B, c, sigmoid)
            assert torch_equal(got["h_last"][0], c["h0"][0]) and torch_equal(got["dh0"][0], c["dl"][0])
            assert (got["y"][0] == 0).all() and (got["dx"][0] == 0).all() and (got["dgate"][0] == 0).all()


def torch_equal(a, b):
    import torch
    return torch.equal(a, b)


def test_no_state_given(B):
    c = case("float32", 2, 200, 24, 1, 3, True, state=False)
    check(B, c, True)


@pytest.mark.parametrize("sigmoid", [True, False])
def test_resets_and_lengths_stop_nan_and_inf(B, sigmoid):
    import torch
    for steps in (6, 300):
        c = case("float32", 3, steps, 34, 1, 2, sigmoid)
        c["reset"] = torch.zeros(3, steps, dtype=torch.uint8, device="cuda")
        c["lengths"] = torch.tensor([steps, steps - 2, 3], dtype=torch.int32, device="cuda")
        want = run(B, c, sigmoid)
        # steps at and beyond a length are not read
        c["x"][1, -2:] = math.nan
        c["gate"][1, -2:] = math.inf
        c["dy"][1, -1] = math.nan
        c["x"][2, 3:] = math.nan
        got = run(B, c, sigmoid)
        for k in want:
            assert torch.equal(want[k], got[k]), k
        # a reset cuts off whatever the state holds
        c["reset"][0, 2] = 1
        want = run(B, c, sigmoid)
        c["h0"][0, :17] = math.inf
        c["h0"][0, 17:] = math.nan
        got = run(B, c, sigmoid)
        assert torch.equal(want["y"][0, 2:], got["y"][0, 2:]) and torch.equal(want["h_last"], got["h_last"])
        assert torch.equal(want["dx"][:, 2:], got["dx"][:, 2:])
        assert torch.equal(want["dgate"][:, 2:], got["dgate"][:, 2:])
        # without one, NaN reaches the end of its own channel and sequence alone
        c = case("float32", 2, steps, 34, 1, 2, sigmoid)
        c["x"][0, 1, 5] = math.nan
        y = run(B, c, sigmoid)["y"]
        bad = y.isnan()
        assert bad[0, 1:, 5].all() and int(bad.sum()) == steps - 1


def test_extreme_gates(B):
    import torch
    x = torch.randn(2, 150, 32, device="cuda")
    gate = torch.full_like(x, 200.0)
    gate[1] = -200.0
    h0 = torch.randn(2, 32, device="cuda")
    r = B.adapt_gated_scan(x, gate, h0=h0, want_carry=True)
    assert torch.equal(r.h_last[0], h0[0])            # the state is held
    assert torch.allclose(r.y[1], x[1], rtol=2.0 ** -20, atol=0)   # the input passes
    g = B.adapt_gated_scan_backward(x, gate, torch.ones_like(x), r.carry, want_dh0=True)
    assert g.dx.isfinite().all() and g.dgate.isfinite().all() and torch.equal(g.dh0[0], torch.full_like(g.dh0[0], 150.0))
    # decays of 0 and of one: sums and copies
    one = torch.ones(1, 1000, 8, device="cuda")
    assert torch.equal(B.adapt_gated_scan(one, one, mode=B.GATE_VALUE).y[0, :, 0], torch.arange(1, 1001, device="cuda").float())
    assert torch.equal(B.adapt_gated_scan(x, torch.zeros_like(x), mode=B.GATE_VALUE).y, x)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(B, dtype):
    import torch
    for steps, channels in ((5, 33), (200, 64), (150, 70)):
        c = case(dtype, 3, steps, channels, 1, 1, True)
        want = run(B, c, True)
        # time-major storage, and slices of a wider buffer
        wide = torch.zeros(3, steps, 3 * channels + 5, dtype=c["x"].dtype, device="cuda")
        wide[..., 1:1 + channels], wide[..., 1 + channels:1 + 2 * channels] = c["x"], c["gate"]
        v = dict(c, x=wide[..., 1:1 + channels], gate=wide[..., 1 + channels:1 + 2 * channels],
                 dy=c["dy"].transpose(0, 1).contiguous().transpose(0, 1))
        out = torch.full((steps, 3, channels + 3), 7.0, dtype=c["x"].dtype, device="cuda")
        y = out.transpose(0, 1)[..., 2:2 + channels]
        r = B.adapt_gated_scan(v["x"], v["gate"], h0=v["h0"], want_carry=True, y=y)
        assert torch.equal(y, want["y"]) and (out[..., :2] == 7).all() and (out[..., -1] == 7).all()
        gx, gg = torch.full_like(out, 7.0), torch.full_like(out, 7.0)
        g = B.adapt_gated_scan_backward(v["x"], v["gate"], v["dy"], r.carry, dh_last=v["dl"], want_dh0=True,
                                        dx=gx.transpose(0, 1)[..., 1:1 + channels],
                                        dgate=gg.transpose(0, 1)[..., 3:3 + channels])
        assert torch.equal(g.dx, want["dx"]) and torch.equal(g.dgate, want["dgate"]) and torch.equal(g.dh0, want["dh0"])
        assert (gx[..., :1] == 7).all() and (gx[..., 1 + channels:] == 7).all() and (gg[..., :3] == 7).all()
        # an input of stride 0 (one row of gates for all steps)
        row = c["gate"][:, :1].expand(3, steps, channels)
        a = B.adapt_gated_scan(c["x"], row, h0=c["h0"]).y
        assert torch.equal(a, B.adapt_gated_scan(c["x"], row.contiguous(), h0=c["h0"]).y)


def test_in_place_state_and_other_stream(B):
    import torch
    for steps in (1, 3, 700):
        c = case("bfloat16", 2, steps, 96, 1, 5, True)
        want = run(B, c, True)
        state, x = c["h0"].clone(), c["x"].clone()
        r = B.adapt_gated_scan(x, c["gate"], h0=state, h_last=state, y=x)
        assert torch.equal(state, want["h_last"]) and torch.equal(x, want["y"])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        r = B.adapt_gated_scan(c["x"], c["gate"], h0=c["h0"], want_carry=True, stream=s)
        dy = c["dy"].clone()
        s.wait_stream(torch.cuda.current_stream())
        g = B.adapt_gated_scan_backward(c["x"], c["gate"], dy, r.carry, dh_last=c["dl"], dx=dy, stream=s)
        s.synchronize()
        assert torch.equal(r.y, want["y"]) and torch.equal(g.dx, want["dx"]) and g.dx is dy


def test_steps_continue_a_sequence(B):
    import torch
    c = case("float32", 2, 260, 64, 1, 9, True)
    whole = B.adapt_gated_scan(c["x"], c["gate"], h0=c["h0"])
    state = c["h0"].clone()
    head = B.adapt_gated_scan(c["x"][:, :250].contiguous(), c["gate"][:, :250].contiguous(), h0=state, h_last=state)
    ys = [head.y]
    for t in range(250, 260):     # one token at a time
        ys.append(B.adapt_gated_scan(c["x"][:, t:t + 1].contiguous(), c["gate"][:, t:t + 1].contiguous(), h0=state, h_last=state).y)
    assert torch.allclose(torch.cat(ys, 1), whole.y, rtol=1e-5, atol=1e-5)
    assert torch.allclose(state, whole.h_last, rtol=1e-5, atol=1e-5)


def test_gradient_against_differences(B):
    import torch
    eps = 2.0 ** -7
    for sigmoid in (True, False):
        c = case("float32", 2, 140, 20, 2, 4, sigmoid, resets=True)
        if not sigmoid:
            c["gate"].mul_(0.9)
        mode = B.GATE_SIGMOID if sigmoid else B.GATE_VALUE
        g = torch.Generator(device="cuda").manual_seed(1)
        v = {k: torch.randn(c[k].shape, generator=g, device="cuda") * 0.1 for k in ("x", "gate", "h0")}

        def value(s):
            r = B.adapt_gated_scan(c["x"] + s * v["x"], c["gate"] + s * v["gate"], h0=c["h0"] + s * v["h0"],
                                   reset=c["reset"], mode=mode)
            return (r.y.double() * c["dy"].double()).sum() + (r.h_last.double() * c["dl"].double()).sum()

        d = (value(eps) - value(-eps)) / (2 * eps)
        got = run(B, c, sigmoid)
        want = sum((got[n].double() * v[k].double()).sum() for n, k in (("dx", "x"), ("dgate", "gate"), ("dh0", "h0")))
        # 5600 products of order 3 with errors of 2^-22 that add like a random walk (times 5); truncation of order eps^2
        size = (got["y"].double().abs() * c["dy"].double().abs()).sum()
        tol = 5 * 2.0 ** -22 * float(size) / 5600 ** 0.5 / eps + eps ** 2 * float(size) * 0.1
        assert abs(d - want) <= tol, (float(d), float(want), tol)


def test_repeated_calls_give_the_same_bits(B):
    import torch
    c = case("bfloat16", 2, 3000, 128, 64, 6, True, resets=True)
    first = run(B, c, True)
    for _ in range(5):
        again = run(B, c, True)
        for k in first:
            assert torch.equal(first[k], again[k]), k


def test_graph_capture_and_changed_inputs(B):
    import torch
    c = case("float32", 1, 2000, 64, 1, 6, True)
    ws_f = B.adapt_gated_scan(c["x"], c["gate"], h0=c["h0"])   # warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = B.adapt_gated_scan(c["x"], c["gate"], h0=c["h0"], want_carry=True)
        g = B.adapt_gated_scan_backward(c["x"], c["gate"], c["dy"], r.carry, dh_last=c["dl"])
    for seed in (1, 2):
        n = case("float32", 1, 2000, 64, 1, seed, True)
        for k in ("x", "gate", "dy", "h0", "dl"):
            c[k].copy_(n[k])
        graph.replay()
        torch.cuda.synchronize()
        want = run(B, c, True)
        assert torch.equal(r.y, want["y"]) and torch.equal(g.dx, want["dx"]) and torch.equal(g.dgate, want["dgate"])
    del ws_f


# About 500 chains of 64 channels: one CTA each on 148 SMs, so the state goes from tile to tile inside the CTA.
# 4000 channels move 16 bytes at a time, 3998 two channels (16-bit: 4-byte rows), 3999 one.
@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype,channels,group", [("bfloat16", 4000, 1), ("float16", 3998, 1), ("bfloat16", 3999, 1),
                                                  ("float32", 4000, 1), ("float32", 3999, 1), ("float16", 4096, 8),
                                                  ("bfloat16", 4096, 64), ("float32", 4096, 128)])
def test_many_chains_run_through_their_tiles(B, sigmoid, dtype, channels, group):
    steps = 150     # two whole tiles and 22 steps
    check(B, case(dtype, 8, steps, channels, group, channels + group, sigmoid), sigmoid)
    lengths = [0, 1, steps, steps - 1, 64, 65, 128, 127]
    c = case(dtype, 8, steps, channels, group, channels, sigmoid, lengths=lengths, resets=True)
    c["reset"][2, 64] = c["reset"][2, 127] = True      # at a tile's first and last step
    check(B, c, sigmoid)


# Few chains: narrower blocks in clusters, over several rounds of exchange (on 148 SMs 32 channels by 8 CTAs, 16
# channels by 16 CTAs, and 64 channels by 16 CTAs with the gate of 64 channels).
@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype,batch,steps,channels,group", [
    ("bfloat16", 2, 9001, 512, 1), ("float32", 2, 9001, 510, 1), ("float16", 2, 9001, 511, 1), ("bfloat16", 1, 9100, 256, 1),
    ("float32", 1, 9100, 250, 2), ("float16", 1, 9100, 256, 64)])
def test_few_chains_run_through_their_rounds(B, sigmoid, dtype, batch, steps, channels, group):
    c = case(dtype, batch, steps, channels, group, steps + group, sigmoid, lengths=[steps, steps - 4000][:batch], resets=True)
    if not sigmoid:
        c["gate"] = c["gate"].clamp(-1, 1)      # (longer products of decays than in the cases above)
    check(B, c, sigmoid)
    check(B, dict(c, reset=None, lengths=None), sigmoid)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("batch,steps,channels", [(2, 16, 64), (2, 17, 64), (2, 40, 33), (1, 300, 64), (1, 9000, 64),
                                                  (8, 130, 4000)])
def test_zero_states_stay_zero_under_large_decays(B, dtype, batch, steps, channels):
    import torch
    big = 3e4 if dtype == "float16" else 1e25      # eight of them (fp16: ten) pass the range of fp32
    gate = torch.full((batch, steps, channels), big, dtype=getattr(torch, dtype), device="cuda")
    zero = torch.zeros_like(gate)
    for at in ([7], [9, 15], list(range(5, steps, 6)), []):
        g = gate.clone()
        for t in at:
            g[:, t] = 0
        r = B.adapt_gated_scan(zero, g, h0=torch.zeros(batch, channels, device="cuda"), mode=B.GATE_VALUE, want_carry=True)
        b = B.adapt_gated_scan_backward(zero, g, zero, r.carry, mode=B.GATE_VALUE, want_dh0=True)
        for name, v in (("y", r.y), ("h_last", r.h_last), ("carry", r.carry), ("dx", b.dx), ("dgate", b.dgate), ("dh0", b.dh0)):
            assert (v == 0).all(), (name, at)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("batch,steps,channels,group", [(2, 6, 32, 1), (2, 40, 32, 1), (1, 300, 96, 4), (1, 2500, 64, 1),
                                                        (8, 150, 4000, 1)])
def test_decays_at_a_reset_do_not_count(B, dtype, batch, steps, channels, group):
    import torch
    c = case(dtype, batch, steps, channels, group, steps, False)
    c["reset"] = torch.zeros(batch, steps, dtype=torch.bool, device="cuda")
    at = [t for t in (0, 3, 5, 12, 31, 64, 130, 131, steps - 1) if t < steps]
    c["reset"][:, at] = True
    want = run(B, c, False)
    for bad in (math.nan, math.inf, -math.inf, 0.0):
        gate = c["gate"].clone()
        gate[:, at] = bad
        got = run(B, dict(c, gate=gate), False)
        for name in want:
            assert torch.equal(got[name], want[name]), (name, bad)


def test_capture_needs_a_workspace_of_the_call_s_own(B):
    import torch
    c = case("float32", 2, 70, 256, 128, 6, True)
    want = run(B, c, True)
    carry = B.adapt_gated_scan(c["x"], c["gate"], h0=c["h0"], want_carry=True).carry
    dx, dgate = torch.zeros_like(c["x"]), torch.zeros_like(c["gate"])
    need = B.adapt_gated_scan_workspace_bytes(2, 70, 256, 128, B.DTYPE_F32, backward=True)
    assert need > 0 and B.adapt_gated_scan_workspace_bytes(2, 70, 256, 64, B.DTYPE_F32, backward=True) == 0
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")

    def call(workspace, size, stream):
        return B.lib().adapt_gated_scan_backward(c["x"].data_ptr(), c["gate"].data_ptr(), c["dy"].data_ptr(), carry.data_ptr(),
                                                 c["dl"].data_ptr(), None, None, 2, 70, 256, 128, B.DTYPE_F32, B.GATE_SIGMOID,
                                                 None, dx.data_ptr(), dgate.data_ptr(), None, workspace, size, stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stream = torch.cuda.current_stream().cuda_stream
        assert call(None, 0, stream) == B.ERR_INVALID_ARG and b"captured" in B.lib().adapt_last_error()
        assert call(scratch.data_ptr(), need - 1, stream) == B.ERR_WORKSPACE
        assert call(scratch.data_ptr(), need, stream) == B.OK
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dx, want["dx"]) and torch.equal(dgate, want["dgate"])
    dgate.zero_()
    assert call(None, 0, torch.cuda.current_stream().cuda_stream) == B.OK      # outside a capture: the library's buffer
    torch.cuda.synchronize()
    assert torch.equal(dgate, want["dgate"])
