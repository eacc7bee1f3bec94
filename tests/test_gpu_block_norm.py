"""Norms before and after a block, with gate and residual, against their definitions in 64 bits."""
import itertools
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2107_13490_b200 import binding as B  # noqa: E402
from tests import layers_reference as R  # noqa: E402

TYPES = [torch.float32, torch.float16, torch.bfloat16]
NONE, RMS, LAYER = B.NORM_NONE, B.NORM_RMS, B.NORM_LAYER
EPS = 1e-5


def make(rows, dim, dtype, gate="each", residual=True, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    v = {"block": (rand(rows, dim) * spread + 0.25).to(dtype), "residual": (rand(rows, dim) * 2).to(dtype) if residual else None,
         "gate": {"none": None, "each": rand(rows, dim).to(dtype) * 2, "shared": rand(dim)}[gate],
         "weight_after": rand(dim) * 0.5 + 1, "weight_before": rand(dim) * 0.5 + 1}
    return v, rand(rows, dim).to(dtype), rand(rows, dim).to(dtype)


def check(v, d_y, d_n, after, before, mode=B.GATE_SIGMOID, scale=0.5, residual_scale=1.25, eps=EPS, backward=True):
    v = dict(v)
    if after == NONE:
        v["weight_after"] = None
    if before == NONE:
        v["weight_before"] = d_n = None
    dtype = v["block"].dtype
    how = dict(**v, after=after, before=before, gate_mode=mode, scale=scale, residual_scale=residual_scale, eps=eps)
    block = how.pop("block")
    r = B.adapt_block_norm(block, want_stats=True, **how)
    dim = block.shape[-1]
    flat = {n: t.reshape(-1, dim) if t is not None and t.dim() > 1 else t for n, t in v.items()}
    ref = R.Norms(flat["block"], flat["residual"], flat["gate"], v["weight_after"], v["weight_before"], after, before, mode == B.GATE_SIGMOID,
                  scale, residual_scale, eps, *((None if d is None else d.reshape(-1, dim)) for d in (d_y, d_n)))
    names = [("y", r.y)] + ([("normed", r.normed)] if before != NONE else [])
    assert before != NONE or r.normed is None
    if backward:
        g = B.adapt_block_norm_backward(block, r.stats, d_y=d_y, d_normed=d_n, **how)
        names += [(n, getattr(g, n)) for n in g.__slots__ if getattr(g, n) is not None]
        again = B.adapt_block_norm_backward(block, r.stats, d_y=d_y, d_normed=d_n, **how)
        for n in g.__slots__:
            assert (getattr(g, n) is None) == (getattr(again, n) is None)
            assert getattr(g, n) is None or torch.equal(getattr(g, n), getattr(again, n)), n
        given = {"d_block": True, "d_residual": v["residual"] is not None, "d_gate": v["gate"] is not None, "d_weight_after": after != NONE,
                 "d_weight_before": before != NONE and d_n is not None}
        assert {n for n, there in given.items() if there} == {n for n, _ in names if n.startswith("d_")}
    for n, got in names:
        want, tol = getattr(ref, n), getattr(ref, n + "_tol")
        assert R.within(got.reshape(want.shape), want, tol + R.half_step(want, got.dtype)), n
    return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("after,before,gate,residual", list(itertools.product((NONE, RMS, LAYER), (NONE, RMS, LAYER), ("none", "each", "shared"),
                                                                              (False, True))))
def test_every_form(dtype, after, before, gate, residual):
    for mode in (B.GATE_SIGMOID, B.GATE_VALUE):
        v, d_y, d_n = make(37, 200, dtype, gate, residual)
        check(v, d_y, d_n, after, before, mode)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("rows,dim", [(1, 8), (3, 33), (2, 64), (1000, 128), (5, 1000), (70, 1024), (700, 1001), (9, 2048), (4, 4096), (150, 4104),
                                      (3, 8192), (2, 8200), (2, 16384), (2, 20001), (2, 32768)])
def test_sizes(dtype, kind, rows, dim):
    v, d_y, d_n = make(rows, dim, dtype)
    check(v, d_y, d_n, kind, kind)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("after,before,gate", [(RMS, LAYER, "each"), (LAYER, NONE, "shared"), (NONE, RMS, "none")])
@pytest.mark.parametrize("rows,dim", [(9999, 72), (4999, 1000), (4997, 1001), (3001, 2040), (3001, 2047), (1201, 4096)])
def test_many_rows(dtype, after, before, gate, rows, dim):
    """Each CTA walks over several rounds of its ring of stages, with a last round of one row or two."""
    v, d_y, d_n = make(rows, dim, dtype, gate)
    check(v, d_y, d_n, after, before)


@pytest.mark.parametrize("dim", [1, 2, 3, 5, 7])
def test_narrowest_rows(dim):
    for after, before in ((RMS, LAYER), (LAYER, RMS), (NONE, RMS), (LAYER, NONE)):
        v, d_y, d_n = make(500, dim, torch.float32)
        check(v, d_y, d_n, after, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(5, 40), (33, 1024), (9, 4096), (3, 9000)])
def test_layouts(dtype, rows, dim):
    """Slices of wider buffers, rows that are the same for all (stride 0), outputs in place."""
    v, d_y, d_n = make(rows, dim, dtype)
    plain = check(v, d_y, d_n, RMS, RMS)
    how = dict(after=RMS, before=RMS, scale=0.5, residual_scale=1.25, eps=EPS, want_stats=True)
    for at in (0, 1, 8):
        sliced = {}
        for n in ("block", "residual", "gate"):
            buf = torch.zeros((rows, dim + 24), dtype=dtype, device="cuda")
            sliced[n] = buf[:, at:at + dim]
            sliced[n].copy_(v[n])
        out = torch.full((2, rows, dim + 24), 3.0, dtype=dtype, device="cuda")
        y, normed = out[0][:, at:at + dim], out[1][:, 8:8 + dim]
        r = B.adapt_block_norm(**{**v, **sliced}, **how, y=y, normed=normed)
        wide = (torch.finfo(dtype).eps / 2 + 2.0 ** -18) * 2      # (another order of the sums)
        for a, b in ((r.y, plain.y), (r.normed, plain.normed)):
            assert torch.allclose(a.float(), b.float(), rtol=wide, atol=wide * 16)
        assert (out[0][:, :at] == 3).all() and (out[0][:, at + dim:] == 3).all() and (out[1][:, :8] == 3).all() and (out[1][:, 8 + dim:] == 3).all()
        check({**v, **sliced}, d_y, d_n, RMS, RMS)
    same = {**v, "residual": v["residual"][:1].expand(rows, dim), "gate": v["gate"][:1].expand(rows, dim)}
    check(same, d_y, d_n, RMS, RMS)
    for n in ("block", "residual", "gate"):     # y over an input
        copy = {**v, n: v[n].clone()}
        r = B.adapt_block_norm(**copy, **how, y=copy[n])
        assert torch.equal(r.y, plain.y) and r.y.data_ptr() == copy[n].data_ptr() and torch.equal(r.normed, plain.normed)
    copy = {**v, "block": v["block"].clone()}   # normed over an input
    assert torch.equal(B.adapt_block_norm(**copy, **how, normed=copy["block"]).normed, plain.normed)
    d = d_y.clone()                             # d_residual over d_y
    back = dict(stats=plain.stats, d_normed=d_n, **v, **{k: how[k] for k in ("after", "before", "scale", "residual_scale", "eps")})
    want = B.adapt_block_norm_backward(d_y=d_y, **back)
    got = B.adapt_block_norm_backward(d_y=d, d_residual=d, **back)
    assert got.d_residual.data_ptr() == d.data_ptr()
    for n in want.__slots__:
        assert torch.equal(getattr(got, n), getattr(want, n)), n


def test_norm_alone_and_parts():
    v, d_y, d_n = make(50, 256, torch.bfloat16, "none", False)
    r = B.adapt_block_norm(v["block"], weight_before=v["weight_before"], want_y=False, want_stats=True)
    assert r.y is None
    ref = R.Norms(v["block"], None, None, None, v["weight_before"], 0, 1, False, 1.0, 1.0, 1e-6, None, d_n)
    assert R.within(r.normed, ref.normed, ref.normed_tol + R.half_step(ref.normed, torch.bfloat16))
    g = B.adapt_block_norm_backward(v["block"], r.stats, d_normed=d_n, weight_before=v["weight_before"], want_weights=False)
    assert g.d_weight_before is None and R.within(g.d_block, ref.d_block, ref.d_block_tol + R.half_step(ref.d_block, torch.bfloat16))
    v, d_y, d_n = make(50, 256, torch.bfloat16)
    for a, b in ((d_y, None), (None, d_n)):     # either gradient alone
        check(v, a, b, RMS, RMS)
    cube = {n: t.reshape(5, 10, 256) if t is not None and t.dim() == 2 else t for n, t in v.items()}
    check(cube, d_y.reshape(5, 10, 256), d_n.reshape(5, 10, 256), LAYER, RMS)


def test_without_weights():
    v, d_y, d_n = make(50, 256, torch.float32)
    v["weight_after"] = v["weight_before"] = None
    for after, before in ((RMS, LAYER), (LAYER, RMS)):
        how = dict(after=after, before=before, eps=EPS, residual=v["residual"], gate=v["gate"])
        r = B.adapt_block_norm(v["block"], want_stats=True, **how)
        g = B.adapt_block_norm_backward(v["block"], r.stats, d_y=d_y, d_normed=d_n, **how)
        assert g.d_weight_after is None and g.d_weight_before is None
        ref = R.Norms(v["block"], v["residual"], v["gate"], None, None, after, before, True, 1.0, 1.0, EPS, d_y, d_n)
        for n, got in (("y", r.y), ("normed", r.normed), ("d_block", g.d_block), ("d_residual", g.d_residual), ("d_gate", g.d_gate)):
            assert R.within(got, getattr(ref, n), getattr(ref, n + "_tol") + R.half_step(getattr(ref, n), torch.float32)), n


def test_far_gates_and_large_means():
    v, d_y, d_n = make(40, 512, torch.float32)
    v["gate"] = torch.linspace(-120, 120, 40 * 512, device="cuda").reshape(40, 512)
    check(v, d_y, d_n, RMS, RMS)
    v, d_y, d_n = make(40, 512, torch.float32)
    v["block"] += 300.0       # a mean far beyond the deviation: the variance is taken around it
    check(v, d_y, d_n, LAYER, LAYER)


@pytest.mark.parametrize("dim", [96, 1001, 4096, 12000])
def test_rows_with_nan_or_infinity_stay_alone(dim):
    v, d_y, d_n = make(12, dim, torch.float32)
    how = dict(after=RMS, before=LAYER, eps=EPS, want_stats=True)
    want = B.adapt_block_norm(**v, **how)
    v["block"][3, dim // 2], v["residual"][7, 0], v["gate"][9, 5] = math.nan, math.inf, math.nan
    got = B.adapt_block_norm(**v, **how)
    clean = [i for i in range(12) if i not in (3, 7, 9)]
    assert torch.equal(got.y[clean], want.y[clean]) and torch.equal(got.normed[clean], want.normed[clean])
    assert got.y[3].isnan().all() and all(got.normed[i].isnan().all() for i in (3, 7, 9))
    zero = torch.zeros(3, dim, device="cuda")
    assert (B.adapt_block_norm(zero, before=RMS, eps=1e-6).normed == 0).all() and (B.adapt_block_norm(zero, before=LAYER, eps=1e-6).normed == 0).all()


def test_no_rows():
    none = torch.zeros(0, 16, device="cuda")
    w = torch.ones(16, device="cuda")
    r = B.adapt_block_norm(none, weight_before=w, want_stats=True)
    assert r.y.shape == r.normed.shape == (0, 16)
    g = B.adapt_block_norm_backward(none, r.stats, d_normed=none, weight_before=w)
    assert (g.d_weight_before == 0).all() and g.d_block.shape == (0, 16)


def test_gradient_against_differences():
    """fp32 forward passes at v +- h d: their difference by 2h is the slope but for h^2 times the third derivative (of
    the order of the slope's terms here) and the forward pass's own tolerance by h."""
    v, d_y, d_n = make(30, 300, torch.float32)
    how = dict(after=LAYER, before=RMS, scale=0.5, residual_scale=1.25, eps=EPS)
    r = B.adapt_block_norm(**v, **how, want_stats=True)
    g = B.adapt_block_norm_backward(stats=r.stats, d_y=d_y, d_normed=d_n, **v, **how)
    ref = R.Norms(v["block"], v["residual"], v["gate"], v["weight_after"], v["weight_before"], LAYER, RMS, True, 0.5, 1.25, EPS, d_y, d_n)
    forward_tol = float((d_y.double().abs() * ref.y_tol).sum() + (d_n.double().abs() * ref.normed_tol).sum())
    h = 2.0 ** -7
    for n in ("block", "residual", "gate", "weight_after", "weight_before"):
        gen = torch.Generator(device="cuda").manual_seed(4)
        d = torch.randn(v[n].shape, generator=gen, device="cuda")
        value = []
        for s in (1, -1):
            f = B.adapt_block_norm(**{**v, n: v[n] + s * h * d}, **how)
            value.append((f.y.double() * d_y.double()).sum() + (f.normed.double() * d_n.double()).sum())
        terms = float((getattr(g, "d_" + n).double().abs() * d.double().abs()).sum())
        want = (getattr(g, "d_" + n).double() * d.double()).sum()
        assert abs((value[0] - value[1]) / (2 * h) - want) <= forward_tol / h + h * h * terms + 4 * R.U * terms, n


def test_streams_and_graphs():
    v, d_y, d_n = make(300, 512, torch.bfloat16)
    how = dict(after=RMS, before=RMS, eps=EPS)

    def both():
        r = B.adapt_block_norm(**v, **how, want_stats=True)
        g = B.adapt_block_norm_backward(stats=r.stats, d_y=d_y, d_normed=d_n, **v, **how)
        return [r.y, r.normed] + [getattr(g, n) for n in g.__slots__]

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both()
        graphs.append((graph, out))
    v["block"].mul_(0.5).add_(0.125)
    for graph, _ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    want = both()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    v, d_y, d_n = make(6, 40, torch.float32)
    x, w = v["block"], v["weight_after"]
    stats = B.adapt_block_norm(x, want_stats=True).stats
    for call in (lambda: B.adapt_block_norm(x.double()), lambda: B.adapt_block_norm(x, residual=x[:5]), lambda: B.adapt_block_norm(x, residual=x.half()),
                 lambda: B.adapt_block_norm(x, gate=x[:, :39]), lambda: B.adapt_block_norm(x, gate=w.half()), lambda: B.adapt_block_norm(x, weight_before=w[:39]),
                 lambda: B.adapt_block_norm(x, weight_before=w.cpu()), lambda: B.adapt_block_norm(x.t()), lambda: B.adapt_block_norm(x, y=x[:5]),
                 lambda: B.adapt_block_norm(x, want_y=False, y=x), lambda: B.adapt_block_norm_backward(x, stats[:5], d_y=d_y),
                 lambda: B.adapt_block_norm_backward(x, stats, d_y=d_y.half()), lambda: B.adapt_block_norm_backward(x, stats, d_y=d_y, d_residual=d_y)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: B.adapt_block_norm(x, after=3), lambda: B.adapt_block_norm(x, weight_after=w), lambda: B.adapt_block_norm(x, eps=-1.0),
                 lambda: B.adapt_block_norm(x, scale=math.nan), lambda: B.adapt_block_norm(x, gate=x, gate_mode=5),
                 lambda: B.adapt_block_norm(x, before=NONE, want_y=False), lambda: B.adapt_block_norm_backward(x, stats),
                 lambda: B.adapt_block_norm(torch.zeros(2, B.NORM_MAX_DIM + 1, device="cuda"))):
        with pytest.raises(B.AdaptError) as e:
            call()
        assert e.value.status == B.ERR_INVALID_ARG
