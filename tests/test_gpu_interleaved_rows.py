"""Inputs and outputs whose rows lie between one another's in one buffer: they share no memory, and
the calls give what they give apart."""
import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from test_gpu_experts import DT, check_sort, choices
from test_gpu_hidden import Plain, backward, inputs

pytestmark = pytest.mark.gpu


def beside(a, b):
    """a and b (as many rows each) as the halves of one buffer's rows."""
    n = max(len(a), len(b))
    buf = torch.full((n, a.shape[1] + b.shape[1]), 5.0, dtype=a.dtype, device="cuda")
    x, y = buf[:len(a), :a.shape[1]], buf[:len(b), a.shape[1]:]
    x.copy_(a), y.copy_(b)
    return x, y


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [24, 61, 256])
def test_rows_of_experts(dtype, D):
    T, k, E = 300, 3, 9
    idx = choices(1, T, k, E)
    place = check_sort(idx, E)[2]
    x = torch.randn((T, D), device="cuda").to(DT[dtype])
    w = torch.rand((T, k), device="cuda")
    rows = torch.zeros((T * k, D), dtype=x.dtype, device="cuda")
    bt.boute_expert_dispatch(x, place, rows)
    a, b = beside(x, torch.zeros_like(rows))
    bt.boute_expert_dispatch(a, place, b)
    assert torch.equal(a, x) and torch.equal(b, rows)
    out = torch.zeros_like(x)
    bt.boute_expert_combine(rows, place, w, out)
    a, b = beside(torch.zeros_like(x), rows)
    bt.boute_expert_combine(b, place, w, a)
    assert torch.equal(a, out) and torch.equal(b, rows)
    go = torch.randn((T, D), device="cuda").to(x.dtype)
    g, gw = torch.zeros_like(rows), torch.zeros_like(w)
    bt.boute_expert_combine_grad(go, rows, place, w, g, gw)
    a, b = beside(rows, torch.zeros_like(rows))
    gw2 = torch.zeros_like(w)
    bt.boute_expert_combine_grad(go, a, place, w, b, gw2)
    assert torch.equal(b, g) and torch.equal(a, rows)
    assert (gw2 - gw).abs().max() <= 1e-4 * (1 + gw.abs().max())  # (lanes' sums by the alignment)


@pytest.mark.parametrize("T,D,dtype", [(40, 64, "f16"), (300, 72, "bf16"), (70, 61, "bf16")])
def test_gradients_beside_the_states_and_the_weight(T, D, dtype):
    h, w, t = inputs(T, 500, D, dtype)
    plain = Plain(h, w, t, 1.0)
    g = torch.randn((T,), device="cuda")
    lse, H = plain.lse.float(), plain.H.float()
    want = backward(h, w, t, 1.0, lse, H, g, g)
    h2, dh = beside(h, torch.zeros_like(h))
    w2, dw = beside(w, torch.zeros_like(w))
    ws = torch.empty((bt.boute_hidden_logprobs_workspace(h2, w2, True),), dtype=torch.uint8, device="cuda")
    bt.boute_hidden_logprobs_grad(h2, w2, t, 1.0, lse, H, g, g, dh, dw, ws)
    assert torch.equal(h2, h) and torch.equal(w2, w)
    assert torch.equal(dh, want[0]) and torch.equal(dw, want[1])
