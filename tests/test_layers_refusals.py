"""Calls of the operators around a language model's layers that the library refuses before anything is launched
(so the pointers below are never followed).  CPU only."""
import ctypes

import pytest
import torch

from paper_2107_13490_b200 import binding as B
from paper_2107_13490_b200 import build

P = 0x10000   # an aligned address
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def embedding(L, **k):
    a = dict(table=P, vocab=10, dim=8, ld=8, dtype=0, ids=P, n=4, scale=1.0, out=P, ldo=8, stream=None)
    a.update(k)
    return L.adapt_embedding(*a.values())


def embedding_backward(L, **k):
    a = dict(dy=P, n=4, dim=8, ld=8, dtype=2, ids=P, vocab=10, scale=1.0, accumulate=0, grad=P, ldg=8, gdtype=2, ws=P, wsn=1 << 20,
             stream=None)
    a.update(k)
    return L.adapt_embedding_backward(*a.values())


def norm_args(**k):
    a = dict(after=1, before=1, gate_mode=0, gate_shared=0, scale=1.0, residual_scale=1.0, eps=1e-6)
    a.update((n, k.pop(n)) for n in list(k) if n in a)
    return B.AdaptNormArgs(*a.values()), k


def norm(L, **k):
    args, k = norm_args(**k)
    a = dict(block=P, residual=P, gate=P, wa=P, wb=P, rows=4, dim=8, dtype=0, args=ctypes.addressof(args), strides=None, y=P, normed=P,
             stats=P, stream=None)
    a.update(k)
    return L.adapt_block_norm(*a.values())


def norm_backward(L, **k):
    args, k = norm_args(**k)
    a = dict(block=P, residual=P, gate=P, wa=P, wb=P, stats=P, d_y=P, d_normed=P, rows=4, dim=8, dtype=0, args=ctypes.addressof(args),
             strides=None, d_block=P, d_residual=P, d_gate=P, dwa=P, dwb=P, ws=P, wsn=1 << 20, stream=None)
    a.update(k)
    return L.adapt_block_norm_backward(*a.values())


def int8_rows(L, **k):
    a = dict(x=P, rows=4, cols=8, ldx=8, dtype=0, codes=P, ldc=8, scales=P, stream=None)
    a.update(k)
    return L.adapt_int8_rows(*a.values())


def int8_linear(L, **k):
    a = dict(x=P, x_dtype=3, xs=P, xsn=4, w=P, ws=P, wsn=6, bias=None, rows=4, n=6, k=8, ldx=8, ldw=8, y=P, ldy=6, dtype=0, work=P,
             workn=1 << 20, stream=None)
    a.update(k)
    return L.adapt_int8_linear(*a.values())


def strides(*v):
    return ctypes.cast((ctypes.c_int64 * len(v))(*v), ctypes.c_void_p)


BIG = 1 << 31


@pytest.mark.parametrize("bad", [
    dict(table=None), dict(ids=None), dict(out=None), dict(vocab=0), dict(vocab=BIG), dict(dim=-1), dict(dim=BIG), dict(n=-1),
    dict(n=BIG), dict(ld=7), dict(ldo=7), dict(dtype=3), dict(dtype=-1), dict(scale=NAN), dict(scale=INF), dict(table=P + 2),
    dict(out=P + 1), dict(ids=P + 4)])
def test_embedding_refuses(L, bad):
    assert embedding(L, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(dy=None), dict(ids=None), dict(grad=None), dict(vocab=0), dict(vocab=BIG), dict(dim=-1), dict(n=-1), dict(n=BIG), dict(ld=7),
    dict(ldg=7), dict(dtype=4), dict(gdtype=1), dict(gdtype=3), dict(dtype=0, gdtype=2), dict(scale=NAN), dict(ws=None), dict(ws=P + 16),
    dict(dy=P + 1), dict(grad=P + 1), dict(gdtype=0, grad=P + 2), dict(ids=P + 4)])
def test_embedding_backward_refuses(L, bad):
    assert embedding_backward(L, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(block=None), dict(rows=-1), dict(rows=BIG), dict(dim=-1), dict(dim=B.NORM_MAX_DIM + 1), dict(dtype=3), dict(args=None), dict(after=3),
    dict(before=-1), dict(gate_mode=2), dict(scale=NAN), dict(residual_scale=INF), dict(eps=-1.0), dict(eps=NAN), dict(after=0),
    dict(before=0), dict(before=0, wb=None), dict(y=None, normed=None), dict(block=P + 2), dict(residual=P + 1), dict(gate=P + 2),
    dict(wa=P + 2), dict(wb=P + 1), dict(y=P + 2), dict(normed=P + 2), dict(stats=P + 8), dict(dtype=2, gate=P + 2, gate_shared=1)])
def test_norm_refuses(L, bad):
    assert norm(L, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(block=None), dict(stats=None), dict(rows=-1), dict(dim=B.NORM_MAX_DIM + 1), dict(dtype=5), dict(args=None), dict(after=0),
    dict(before=0), dict(d_y=None, d_normed=None, dwb=None), dict(d_normed=None), dict(residual=None), dict(gate=None), dict(ws=None),
    dict(ws=P + 128), dict(d_block=P + 2), dict(d_y=P + 1), dict(d_normed=P + 2), dict(d_gate=P + 2), dict(dwa=P + 2), dict(stats=P + 4)])
def test_norm_backward_refuses(L, bad):
    assert norm_backward(L, **bad) == B.ERR_INVALID_ARG


def test_norm_refuses_strides(L):
    for k, v in ((0, 7), (1, -8), (2, 5), (3, 7), (3, 0), (4, 0)):
        s = [8] * 5
        s[k] = v
        assert norm(L, strides=strides(*s)) == B.ERR_INVALID_ARG
    for k, v in ((0, 7), (1, -8), (2, 5), (3, 7), (4, -1), (5, 0), (6, 7), (7, 0)):
        s = [8] * 8
        s[k] = v
        assert norm_backward(L, strides=strides(*s)) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(codes=None), dict(scales=None), dict(rows=-1), dict(cols=-1), dict(rows=BIG), dict(cols=BIG), dict(ldx=7), dict(ldc=7),
    dict(ldc=0), dict(dtype=3), dict(x=P + 2), dict(scales=P + 2)])
def test_int8_rows_refuses(L, bad):
    assert int8_rows(L, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(y=None), dict(rows=-1), dict(n=-1), dict(k=-1), dict(rows=BIG), dict(n=BIG),
    dict(k=B.INT8_MAX_K + 1), dict(ldx=7), dict(ldw=7), dict(ldy=5), dict(ldx=-8), dict(dtype=3), dict(x_dtype=4), dict(xsn=2), dict(wsn=2),
    dict(x_dtype=0), dict(x_dtype=0, xs=None, x=P + 2), dict(x_dtype=0, xs=None, rows=40, work=None),
    dict(x_dtype=2, xs=None, rows=40, work=P + 64),
    dict(y=P + 2), dict(bias=P + 2), dict(xs=P + 1), dict(ws=P + 2)])
def test_int8_linear_refuses(L, bad):
    assert int8_linear(L, **bad) == B.ERR_INVALID_ARG


def test_workspaces_that_are_too_small(L):
    need = B.adapt_embedding_workspace_bytes(4, 8, 10)
    assert need > 0 and embedding_backward(L, wsn=need - 1) == B.ERR_WORKSPACE
    need = B.adapt_block_norm_workspace_bytes(4, 8)
    assert need > 0 and norm_backward(L, wsn=need - 1) == B.ERR_WORKSPACE
    need = B.lib().adapt_int8_linear_workspace_bytes(P, B.DTYPE_BF16, P, 40, 6, 8, 8, 16)
    assert need > 0 and int8_linear(L, rows=40, x_dtype=2, xs=None, ldw=16, workn=need - 1) == B.ERR_WORKSPACE
    more = B.lib().adapt_int8_linear_workspace_bytes(P, B.DTYPE_BF16, P, 40, 6, 8, 8, 8)     # codes between 16-byte boundaries are copied
    assert more > need and int8_linear(L, rows=40, x_dtype=2, xs=None, workn=more - 1) == B.ERR_WORKSPACE


def test_workspace_queries_of_invalid_sizes():
    assert B.adapt_embedding_workspace_bytes(-1, 8, 10) == B.adapt_embedding_workspace_bytes(4, 8, 0) == 0
    assert B.adapt_block_norm_workspace_bytes(0, 8) == B.adapt_block_norm_workspace_bytes(4, B.NORM_MAX_DIM + 1) == 0
    query = B.lib().adapt_int8_linear_workspace_bytes
    assert query(P, 0, P, 40, 6, B.INT8_MAX_K + 1, 1 << 18, 1 << 18) == query(P, 9, P, 40, 6, 8, 8, 8) == 0


def test_sizes_of_zero_are_legal(L):
    assert embedding(L, n=0, ids=None, out=None) == embedding(L, dim=0) == B.OK
    assert embedding_backward(L, dim=0) == embedding_backward(L, n=0, dy=None, ids=None, ws=None, wsn=0, accumulate=1) == B.OK
    assert norm(L, rows=0, block=None) == norm(L, dim=0, block=None) == B.OK
    assert norm_backward(L, dim=0, block=None) == B.OK
    assert norm_backward(L, rows=0, block=None, dwa=None, dwb=None) == B.OK
    assert int8_rows(L, rows=0, x=None, codes=None, scales=None) == B.OK
    assert int8_linear(L, rows=0, xsn=0) == int8_linear(L, n=0, wsn=0) == B.OK


def test_host_tensors_and_other_objects_are_refused():
    m, ids = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int64)
    codes = torch.zeros(3, 4, dtype=torch.int8)
    for call in (lambda: B.adapt_embedding(m, ids), lambda: B.adapt_embedding_backward(m, ids, 5), lambda: B.adapt_block_norm(m),
                 lambda: B.adapt_block_norm_backward(m, m, d_y=m), lambda: B.adapt_int8_rows(m),
                 lambda: B.adapt_int8_linear(m, codes, m[0]), lambda: B.adapt_int8_linear(codes, codes, m[0], x_scales=m[:, 0]),
                 lambda: B.adapt_embedding(None, ids), lambda: B.adapt_block_norm([1.0])):
        with pytest.raises(AssertionError):
            call()
