"""Calls of the training-step operators that the library refuses before anything is launched (so the
pointers below are never followed).  CPU only."""
import ctypes

import pytest

from paper_2107_13490_b200 import binding as B
from paper_2107_13490_b200 import build

P = 0x10000   # an aligned address


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def dropout(L, **k):
    a = dict(x=P, r=None, y=P, rows=4, cols=8, ldx=8, ldr=8, ldy=8, dtype=0, p=0.5, seed=0, layer=0, base=0, stream=None)
    a.update(k)
    return L.adapt_dropout(*a.values())


def logprobs(L, **k):
    a = dict(x=P, rows=4, vocab=10, ld=10, dtype=0, scale=1.0, t=P, top=2, lp=P, ent=P, lse=P, ids=P, tops=P,
             dlp=None, dh=None, dx=None, ldg=0, stream=None)
    a.update(k)
    return L.adapt_token_logprobs(*a.values())


def logprobs_backward(L, **k):
    a = dict(x=P, rows=4, vocab=10, ld=10, dtype=0, scale=1.0, t=P, lse=P, ent=P, dlp=P, dh=P, dx=P, ldg=10, stream=None)
    a.update(k)
    return L.adapt_token_logprobs_backward(*a.values())


def scan(L, **k):
    a = dict(x=P, gate=P, h0=None, lengths=None, reset=None, batch=2, steps=3, channels=64, group=1, dtype=0, mode=0,
             strides=None, y=P, h_last=None, carry=None, ws=None, wsn=0, stream=None)
    a.update(k)
    return L.adapt_gated_scan(*a.values())


def scan_backward(L, **k):
    a = dict(x=P, gate=P, dy=P, carry=P, dh=None, lengths=None, reset=None, batch=2, steps=3, channels=64, group=1,
             dtype=0, mode=0, strides=None, dx=P, dgate=P, dh0=None, ws=None, wsn=0, stream=None)
    a.update(k)
    return L.adapt_gated_scan_backward(*a.values())


def strides(*v):
    return ctypes.cast((ctypes.c_int64 * len(v))(*v), ctypes.c_void_p)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(rows=-1), dict(cols=-1), dict(dtype=3), dict(dtype=-1), dict(p=-0.01),
    dict(p=1.01), dict(p=float("nan")), dict(ldx=7), dict(ldy=7), dict(r=P, ldr=7), dict(x=P + 2), dict(y=P + 1),
    dict(r=P + 2), dict(dtype=2, x=P + 1), dict(rows=1 << 40, cols=1 << 40), dict(base=(1 << 62) + 1)])
def test_dropout_refuses(L, bad):
    assert dropout(L, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(ld=9), dict(dtype=7),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(top=-1), dict(top=33),
    dict(vocab=3, ld=3, top=4), dict(ids=None), dict(tops=None), dict(t=None), dict(t=None, lp=None, dlp=P, dx=P, ldg=10),
    dict(dlp=P), dict(dh=P), dict(dx=P), dict(dlp=P, dx=P, ldg=9), dict(x=P + 1), dict(t=P + 4), dict(lse=P + 2),
    dict(dlp=P, dx=P + 2, ldg=10)])
def test_logprobs_refuses(L, bad):
    assert logprobs(L, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(lse=None), dict(dx=None), dict(dlp=None, dh=None), dict(t=None), dict(ent=None), dict(vocab=0),
    dict(ld=3), dict(ldg=3), dict(scale=0.0), dict(dtype=9), dict(dx=P + 2)])
def test_logprobs_backward_refuses(L, bad):
    assert logprobs_backward(L, **bad) == B.ERR_INVALID_ARG


COMMON = [dict(x=None), dict(gate=None), dict(batch=-1), dict(steps=-1), dict(channels=-1), dict(group=0), dict(group=3),
          dict(group=128), dict(channels=63, group=2), dict(channels=192, group=96), dict(dtype=5), dict(mode=2),
          dict(x=P + 2), dict(gate=P + 1), dict(lengths=P + 2), dict(steps=1 << 31), dict(channels=1 << 31)]


@pytest.mark.parametrize("bad", COMMON + [
    dict(y=None), dict(y=P + 2), dict(h0=P + 2), dict(carry=P + 2), dict(h_last=P + 1)])
def test_scan_refuses(L, bad):
    assert scan(L, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", COMMON + [
    dict(dy=None), dict(carry=None), dict(dx=None), dict(dgate=None), dict(dx=P + 2), dict(dh=P + 2), dict(dh0=P + 2)])
def test_scan_backward_refuses(L, bad):
    assert scan_backward(L, **bad) == B.ERR_INVALID_ARG


def test_scan_refuses_strides(L):
    ok = [192, 64, 192, 64, 192, 64]
    for k, v in ((0, -192), (3, -64), (5, 63), (4, 64)):   # negative inputs, overlapping outputs
        s = list(ok)
        s[k] = v
        assert scan(L, strides=strides(*s)) == B.ERR_INVALID_ARG
    ok = [192, 64] * 5
    for k, v in ((5, -1), (7, 63), (6, 64), (9, 0)):
        s = list(ok)
        s[k] = v
        assert scan_backward(L, strides=strides(*s)) == B.ERR_INVALID_ARG


def test_sizes_of_zero_are_legal(L):
    assert dropout(L, rows=0, x=None, y=None) == B.OK and dropout(L, cols=0) == B.OK
    assert logprobs(L, rows=0) == B.OK and logprobs_backward(L, rows=0) == B.OK
    assert scan(L, batch=0) == B.OK and scan(L, channels=0) == B.OK
    assert scan_backward(L, batch=0) == B.OK


def test_arrays_of_no_rows_need_no_address(L):
    none = dict(rows=0, x=None, t=None)
    assert logprobs(L, **none, lp=None, ent=None, lse=None, ids=None, tops=None) == B.OK
    assert logprobs(L, **none, lp=None, ent=None, lse=None, ids=None, tops=None, dlp=P) == B.OK
    assert logprobs_backward(L, **none, lse=None, ent=None, dlp=None, dh=None, dx=None) == B.OK
    # what does not hang on the rows is still refused
    assert logprobs(L, **none, top=33) == logprobs(L, **none, dtype=4) == logprobs(L, **none, scale=0.0) == B.ERR_INVALID_ARG
    assert logprobs_backward(L, **none, vocab=0) == logprobs_backward(L, **none, scale=-1.0) == B.ERR_INVALID_ARG


def test_workspace_query(L):
    assert B.adapt_gated_scan_workspace_bytes(2, 3, 64) >= 0
    assert B.adapt_gated_scan_workspace_bytes(2, 3, 64, gate_group=3) == 0
    assert B.adapt_gated_scan_workspace_bytes(-2, 3, 64) == 0
