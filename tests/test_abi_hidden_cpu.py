"""Refusals of the entry points over hidden states, before any device call."""
import ctypes

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from test_abi_answers_cpu import BAD, ODD, P, UNS, call, lib  # noqa: F401
from test_abi_answers_devices_cpu import On
from test_abi_experts_cpu import launched  # noqa: F401

WS, Q = ctypes.c_void_p(1 << 20), ctypes.c_void_p(128)
F32, F16, I64, U8 = torch.float32, torch.float16, torch.int64, torch.uint8
COMMON = (dict(h=None), dict(h=ODD), dict(w=None), dict(w=ODD), dict(dt=3), dict(dt=-1), dict(T=-1),
          dict(D=0), dict(V=0), dict(ldh=63), dict(ldw=63))
LIMITS = (dict(dt=0), dict(T=(1 << 20) + 1), dict(V=(1 << 20) + 1),
          dict(D=(1 << 16) + 1, ldh=1 << 17, ldw=1 << 17))


def test_workspace_refusals_and_sizes(lib):  # noqa: F811
    n = ctypes.c_longlong(-1)
    good = dict(h=P, dt=2, T=4, D=64, ldh=64, w=P, V=100, ldw=64, grad=0, n=ctypes.byref(n))
    f = lib.boute_hidden_logprobs_workspace
    for change in COMMON + (dict(n=None),):
        assert call(f, good, **change) == BAD, change
    for change in LIMITS:
        assert call(f, good, **change) == UNS, change

    def size(**change):
        assert call(f, good, **change) == 0
        return n.value

    assert 0 < size() < 1 << 20
    # no logits: 4096 x 131072 of them are 1 GB in 16 bits. Three floats for each half of a tile of 256
    # tokens and each position are 50 MB, an aligned copy of the hidden states 17; the gradient has 256 MB
    # of coefficients at once and up to 128 of dh's sums.
    big = dict(T=4096, D=2048, ldh=2048, V=131072, ldw=2048)
    assert size(**big) < 68 << 20 and size(**big, grad=1) < 512 << 20
    # an aligned copy of what is not
    assert size(ldw=65) >= size() + 100 * 64 * 2
    assert size(T=1, ldh=65) == size(T=1)  # (one row has no pitch)


def test_forward_refusals(lib):  # noqa: F811
    good = dict(h=P, dt=2, T=4, D=64, ldh=64, w=P, V=100, ldw=64, t=P, scale=1.0, lp=P, H=P, lse=P,
                ws=WS, n=1 << 30, s=None)
    f = lib.boute_hidden_logprobs
    for change in COMMON + (dict(t=None), dict(t=ctypes.c_void_p(68)), dict(scale=0.0),
                            dict(scale=float("nan")), dict(scale=float("inf")), dict(lp=None),
                            dict(H=ODD), dict(lse=None), dict(ws=None), dict(ws=P), dict(n=100)):
        assert call(f, good, **change) == BAD, change
    for change in LIMITS:
        assert call(f, good, **change) == UNS, change


def test_gradient_refusals(lib):  # noqa: F811
    good = dict(h=P, dt=1, T=4, D=64, ldh=64, w=P, V=100, ldw=64, t=P, scale=1.0, lse=P, H=P, g=P, gh=P,
                dh=Q, lddh=1 << 17, dw=Q, lddw=1 << 17, ws=WS, n=1 << 30, s=None)
    f = lib.boute_hidden_logprobs_grad
    for change in COMMON + (dict(t=None), dict(scale=-1.0), dict(lse=None), dict(H=None), dict(H=ODD),
                            dict(g=None), dict(gh=ODD), dict(dh=None), dict(dh=ODD), dict(lddh=63),
                            dict(dw=None), dict(dh=P), dict(dw=P), dict(lddw=63), dict(ws=None), dict(ws=P), dict(n=100)):
        assert call(f, good, **change) == BAD, change
    for change in LIMITS:
        assert call(f, good, **change) == UNS, change


def calls(dev):
    at = iter(dev)
    t = lambda *a: On(next(at), *a)
    return [
        (bt.boute_hidden_logprobs, lambda: (t(F16, 4, 9), t(F16, 50, 9), t(I64, 4), 1.0, t(F32, 4),
                                            t(F32, 4), t(F32, 4), t(U8, 999))),
        (bt.boute_hidden_logprobs_grad, lambda: (t(F16, 4, 9), t(F16, 50, 9), t(I64, 4), 1.0, t(F32, 4),
                                                 t(F32, 4), t(F32, 4), t(F32, 4), t(F16, 4, 9),
                                                 t(F16, 50, 9), t(U8, 999))),
    ]


TENSORS = (7, 10)


@pytest.fixture(autouse=True)
def sizes_of_tensors(monkeypatch):
    monkeypatch.setattr(On, "numel", lambda self: self.shape[0], raising=False)
    monkeypatch.setattr(On, "element_size", lambda self: 1, raising=False)


@pytest.mark.parametrize("i", range(len(TENSORS)))
def test_tensors_of_another_device_are_refused(i, launched):  # noqa: F811
    n = TENSORS[i]
    f, args = calls([0] * n)[i]
    f(*args())
    assert launched == [(f.__name__, 100)]
    for odd in range(n):
        for dev in (1, -1):
            f, args = calls([dev if j == odd else 0 for j in range(n)])[i]
            with pytest.raises(ValueError):
                f(*args())
    f, args = calls([1] * n)[i]
    with pytest.raises(ValueError):
        f(*args())
    assert len(launched) == 1


def test_binding_refuses_tensors_that_do_not_fit(launched):  # noqa: F811
    t = lambda *a: On(0, *a)
    good = [t(F16, 4, 9), t(F16, 50, 9), t(I64, 4), 1.0, t(F32, 4), t(F32, 4), t(F32, 4), t(U8, 999)]
    for i, other, error in ((0, t(torch.bfloat16, 4, 9), TypeError), (1, t(F16, 50, 8), ValueError),
                            (2, t(I64, 5), ValueError), (4, t(F32, 3), ValueError),
                            (5, t(F16, 4), TypeError)):
        args = list(good)
        args[i] = other
        with pytest.raises(error):
            bt.boute_hidden_logprobs(*args)
    assert launched == []
