"""Refusals of the entry points over experts' rows, before any device call."""
import ctypes

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from test_abi_answers_cpu import BAD, ODD, P, UNS, call, lib  # noqa: F401
from test_abi_answers_devices_cpu import On

Q, G = ctypes.c_void_p(128), ctypes.c_void_p(192)
H = ctypes.c_void_p(66)  # (aligned to 2 bytes alone)


def test_sort_refusals(lib):  # noqa: F811
    good = dict(idx=P, T=4, k=2, E=9, off=Q, src=Q, place=Q, s=None)
    f = lib.boute_expert_sort
    for change in (dict(idx=None), dict(idx=ODD), dict(T=-1), dict(k=0), dict(E=0), dict(off=None),
                   dict(off=H), dict(src=None), dict(place=H), dict(place=P), dict(src=P)):
        assert call(f, good, **change) == BAD, change
    for change in (dict(k=33), dict(E=1025), dict(T=1 << 30), dict(T=1 << 62)):
        assert call(f, good, **change) == UNS, change


def test_rows_refusals(lib):  # noqa: F811
    good = dict(x=P, dtype=0, T=4, D=10, ldx=10, place=P, k=2, rows=Q, R=8, ldr=12, s=None)
    bad = (dict(dtype=3), dict(dtype=-1), dict(T=-1), dict(D=0), dict(ldx=9), dict(ldr=9), dict(k=0),
           dict(R=-1), dict(place=None), dict(place=H), dict(rows=None), dict(x=None))
    uns = (dict(k=33), dict(T=1 << 30), dict(R=1 << 31), dict(D=(1 << 20) + 1, ldx=1 << 21, ldr=1 << 21))
    f = lib.boute_expert_dispatch
    for change in bad + (dict(x=H), dict(rows=H), dict(rows=P)):
        assert call(f, good, **change) == BAD, change
    for change in uns:
        assert call(f, good, **change) == UNS, change
    good = dict(rows=P, dtype=2, R=8, D=10, ldr=12, place=P, T=4, k=2, x=Q, ldx=10, s=None)
    for change in bad + (dict(x=P),):
        assert call(lib.boute_expert_dispatch_grad, good, **change) == BAD, change
    for change in uns:
        assert call(lib.boute_expert_dispatch_grad, good, **change) == UNS, change
    good = dict(rows=P, dtype=1, R=8, D=10, ldr=12, place=P, w=P, T=4, k=2, x=Q, ldx=10, s=None)
    for change in bad + (dict(w=None), dict(w=H), dict(x=ODD), dict(x=P)):
        assert call(lib.boute_expert_combine, good, **change) == BAD, change
    for change in uns:
        assert call(lib.boute_expert_combine, good, **change) == UNS, change
    good = dict(x=P, dtype=0, T=4, D=10, ldx=10, rows=Q, R=8, ldr=12, place=P, w=P, k=2, g=G, ldg=10,
                gw=P, s=None)
    for change in bad + (dict(w=None), dict(gw=None), dict(gw=H), dict(g=None), dict(g=H), dict(ldg=9),
                         dict(g=P), dict(g=Q)):  # (g_out; in place with another pitch)
        assert call(lib.boute_expert_combine_grad, good, **change) == BAD, change
    for change in uns:
        assert call(lib.boute_expert_combine_grad, dict(good, ldg=1 << 21), **change) == UNS, change


F32, F16, I32 = torch.float32, torch.float16, torch.int32


def calls(dev):
    """(function, arguments) of each call with tensors on device dev[i]."""
    at = iter(dev)
    t = lambda *a: On(next(at), *a)
    return [
        (bt.boute_expert_sort, lambda: (t(I32, 4, 2), t(I32, 9), t(I32, 8), t(I32, 4, 2))),
        (bt.boute_expert_dispatch, lambda: (t(F16, 4, 9), t(I32, 4, 2), t(F16, 8, 9))),
        (bt.boute_expert_dispatch_grad, lambda: (t(F16, 8, 9), t(I32, 4, 2), t(F16, 4, 9))),
        (bt.boute_expert_combine, lambda: (t(F16, 8, 9), t(I32, 4, 2), t(F32, 4, 2), t(F16, 4, 9))),
        (bt.boute_expert_combine_grad, lambda: (t(F16, 4, 9), t(F16, 8, 9), t(I32, 4, 2), t(F32, 4, 2),
                                                t(F16, 8, 9), t(F32, 4, 2))),
    ]


TENSORS = (4, 3, 3, 4, 6)  # of each call


@pytest.fixture
def launched(monkeypatch):
    done = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: done.append((name, a[-1])) or 0

    monkeypatch.setattr(bt, "load", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(bt, "_raw_stream", lambda dev: 100 + dev)
    return done


@pytest.mark.parametrize("i", range(len(TENSORS)))
def test_tensors_of_another_device_are_refused(i, launched):
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


def test_binding_refuses_tensors_that_do_not_fit(launched):
    t = lambda *a: On(0, *a)
    good = [t(F16, 8, 9), t(I32, 4, 2), t(F32, 4, 2), t(F16, 4, 9)]
    for i, other, error in ((0, t(F32, 8, 9), TypeError), (0, t(F16, 8, 10), ValueError),
                            (1, t(I32, 5, 2), ValueError), (1, t(torch.int64, 4, 2), TypeError),
                            (2, t(F32, 4, 3), ValueError), (3, t(torch.float64, 4, 9), TypeError)):
        args = list(good)
        args[i] = other
        with pytest.raises(error):
            bt.boute_expert_combine(*args)
    with pytest.raises(ValueError):
        bt.boute_expert_sort(t(I32, 4, 2), t(I32, 9), t(I32, 7), t(I32, 4, 2))
    assert launched == []
