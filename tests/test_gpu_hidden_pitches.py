"""Gradients of hidden states whose rows have any pitch: one row's is nobody's, and rows may lie more
than 2 GB apart."""
import ctypes

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from test_gpu_hidden import Plain, inputs

pytestmark = pytest.mark.gpu


def call(h, w, t, lse, g, dh, dw, ldh, ldw, lddh, lddw):
    code = {torch.float16: 1, torch.bfloat16: 2}[h.dtype]
    p = lambda x: ctypes.c_void_p(x.data_ptr())
    T, D = h.shape
    n = ctypes.c_longlong()
    lib = bt.load()
    assert lib.boute_hidden_logprobs_workspace(p(h), code, T, D, ldh, p(w), w.shape[0], ldw, 1,
                                               ctypes.byref(n)) == 0
    ws = torch.empty((n.value,), dtype=torch.uint8, device="cuda")
    r = lib.boute_hidden_logprobs_grad(p(h), code, T, D, ldh, p(w), w.shape[0], ldw, p(t), 1.0, p(lse), None,
                                       p(g), None, p(dh), lddh, p(dw), lddw, p(ws), n.value, None)
    torch.cuda.synchronize()
    return r


@pytest.mark.parametrize("T,V,D", [(1, 1, 64), (1, 300, 72), (40, 1, 64), (40, 1, 61)])
@pytest.mark.parametrize("far", [1 << 31, 1 << 45, (1 << 45) + 1])
def test_one_row_has_no_pitch(T, V, D, far):
    h, w, t = inputs(T, V, D, "bf16")
    plain = Plain(h, w, t, 1.0)
    g = torch.randn((T,), device="cuda")
    dh, dw = torch.full_like(h, 5.0), torch.full_like(w, 5.0)
    ld = lambda rows: far if rows == 1 else D
    torch.cuda.synchronize()
    assert call(h, w, t, plain.lse.float(), g, dh, dw, ld(T), ld(V), ld(T), ld(V)) == 0
    a, b, ta, tb = plain.grad(g, None, "bf16")
    assert ((dh.double() - a).abs() <= ta).all() and ((dw.double() - b).abs() <= tb).all()


@pytest.mark.parametrize("T", [0, 40])
@pytest.mark.parametrize("pitch", [(1 << 30) + 8, (1 << 30) + 3])
def test_rows_of_the_weights_gradient_far_apart(T, pitch):
    V, D = 3, 72
    h, w, t = inputs(max(T, 1), V, D, "bf16")
    plain = Plain(h, w, t, 1.0)
    h, t, lse = h[:T], t[:T], plain.lse.float()[:T]
    buf = torch.full(((V - 1) * pitch + D + 8,), 5.0, dtype=torch.bfloat16, device="cuda")
    dw = buf[:(V - 1) * pitch + D].as_strided((V, D), (pitch, 1))
    dh, g = torch.full_like(h, 5.0), torch.ones((T,), device="cuda")
    ws = torch.empty((bt.boute_hidden_logprobs_workspace(h, w, True),), dtype=torch.uint8, device="cuda")
    bt.boute_hidden_logprobs_grad(h, w, t, 1.0, lse, None, g, None, dh, dw, ws)
    assert all((buf[r * pitch + D:r * pitch + D + 8] == 5).all() for r in range(V))
    if T == 0:
        assert not dw.any()
    else:
        a, b, ta, tb = plain.grad(g, None, "bf16")
        assert ((dh.double() - a).abs() <= ta).all() and ((dw.double() - b).abs() <= tb).all()
