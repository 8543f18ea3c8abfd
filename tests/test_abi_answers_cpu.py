"""Refusals of the entry points over a model's answers, before any device call."""
import ctypes

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from paper_2602_10729_gb300 import build as bld

BAD, UNS = bt.BOUTE_ERR_INVALID_ARG, bt.BOUTE_ERR_UNSUPPORTED
P, ODD = ctypes.c_void_p(64), ctypes.c_void_p(65)


@pytest.fixture(scope="module")
def lib():
    bld.build()
    return bt.load()


def call(entry, good, **change):
    return entry(*dict(good, **change).values())


def test_token_logprobs_refusals(lib):
    good = dict(x=P, dtype=2, T=4, V=100, ld=100, t=P, scale=1.0, k=5, lp=P, H=P, lse=P, ti=P, tv=P,
                s=None)
    f = lib.boute_token_logprobs
    for change in (dict(x=None), dict(x=ODD), dict(dtype=3), dict(dtype=-1), dict(T=-1), dict(V=0),
                   dict(ld=99), dict(t=None), dict(t=ctypes.c_void_p(68)), dict(scale=0.0),
                   dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                   dict(k=-1), dict(k=101), dict(lp=None), dict(H=None), dict(lse=ODD),
                   dict(ti=None), dict(tv=None)):
        assert call(f, good, **change) == BAD, change
    for change in (dict(T=1 << 31), dict(V=(1 << 20) + 1, ld=1 << 21), dict(k=33)):
        assert call(f, good, **change) == UNS, change


def test_token_logprobs_grad_refusals(lib):
    Q = ctypes.c_void_p(128)
    good = dict(x=P, dtype=0, T=4, V=100, ld=104, t=P, scale=1.0, lse=P, H=P, g=P, gh=P, dx=Q,
                ldd=100, s=None)
    f = lib.boute_token_logprobs_grad
    for change in (dict(x=None), dict(x=ctypes.c_void_p(66)), dict(dtype=9), dict(ld=99),
                   dict(ldd=99), dict(t=None), dict(lse=None), dict(g=None), dict(H=None),
                   dict(dx=None), dict(scale=0.0), dict(dx=P)):  # (in place with another pitch)
        assert call(f, good, **change) == BAD, change
    assert call(f, good, T=1 << 31) == UNS


def test_answer_scores_refusals(lib):
    good = dict(lp=P, H=P, t=None, off=P, T=10, Q=3, sc=P, n=P, s=None)
    for change in (dict(lp=None), dict(H=ODD), dict(t=ODD), dict(off=None), dict(T=-1), dict(Q=-1),
                   dict(sc=None), dict(n=None)):
        assert call(lib.boute_answer_scores, good, **change) == BAD, change
    assert call(lib.boute_answer_scores, good, T=1 << 31) == UNS
    assert call(lib.boute_answer_scores, good, Q=1 << 31) == UNS
    good = dict(lp=P, H=P, t=None, off=P, T=10, Q=3, g=P, gl=P, gh=P, s=None)
    for change in (dict(g=None), dict(gl=None), dict(gh=None), dict(off=ODD)):
        assert call(lib.boute_answer_scores_grad, good, **change) == BAD, change


def test_route_refusals(lib):
    good = dict(x=P, dtype=2, T=4, E=96, ld=96, b=None, mode=0, G=8, keep=4, gt=2, k=6, rn=1, f=1.0,
                i=P, w=P, l=None, s=None)
    f = lib.boute_route
    for change in (dict(x=None), dict(dtype=5), dict(T=-1), dict(E=0), dict(ld=95), dict(b=ODD),
                   dict(mode=2), dict(mode=-1), dict(G=0), dict(G=7), dict(keep=0), dict(keep=9),
                   dict(gt=0), dict(gt=3), dict(k=0), dict(k=49), dict(f=float("nan")),
                   dict(i=None), dict(w=None), dict(l=ODD)):
        assert call(f, good, **change) == BAD, change
    for change in (dict(E=2048, ld=2048), dict(E=99, ld=99, G=33), dict(keep=8, k=33),
                   dict(T=1 << 31), dict(T=1 << 29)):
        assert call(f, good, **change) == UNS, change
    Q = ctypes.c_void_p(128)
    good = dict(x=P, dtype=1, T=4, E=96, ld=96, mode=1, k=6, rn=1, f=1.0, i=P, g=P, dx=Q, ldd=96,
                s=None)
    f = lib.boute_route_grad
    for change in (dict(x=None), dict(dtype=5), dict(ld=95), dict(ldd=95), dict(mode=2), dict(k=0),
                   dict(k=97), dict(i=None), dict(g=None), dict(dx=None), dict(dx=P, ldd=97)):
        assert call(f, good, **change) == BAD, change
    assert call(f, good, k=33) == UNS


def test_binding_refuses_tensors_that_do_not_fit(lib):
    x = torch.zeros((4, 10))
    t = torch.zeros(4, dtype=torch.int64)
    v = torch.zeros(4)
    with pytest.raises(ValueError):  # not on the device
        bt.boute_token_logprobs(x, t, 1.0, v, v, v)
    with pytest.raises(TypeError):
        bt.boute_token_logprobs(x.double(), t, 1.0, v, v, v)
    with pytest.raises(ValueError):
        bt.boute_token_logprobs(x.t(), t, 1.0, v, v, v)
    with pytest.raises(ValueError):
        bt.boute_token_logprobs(x[:1].expand(4, 10), t, 1.0, v, v, v)
    with pytest.raises(ValueError):
        bt.boute_answer_scores(v, v, t[:3], t, torch.zeros((3, 4)), torch.zeros(3))
