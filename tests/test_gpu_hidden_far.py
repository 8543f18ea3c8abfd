"""Gradients of log-probabilities from hidden states where lse is far from 0: its rounding in fp32
would be in every p. The hidden states' first element times a weight that all tokens share takes the
logits there; the others are small multiples of powers of two, so that all sums are exact."""
import math

import numpy as np
import pytest
import torch

from _answers import U
from paper_2602_10729_gb300 import boute as bt
from test_gpu_hidden import DT, EPS, STEP, TINY, backward, forward

pytestmark = pytest.mark.gpu


def far_inputs(T, V, D, dtype, first, common, seed=0):
    """x = first common + multiples of 1/16 below 2^5."""
    g = torch.Generator(device="cuda").manual_seed(seed + T + V + D)
    grid = lambda *s: torch.randint(-4, 5, s, generator=g, device="cuda") / 4.0
    h, w = grid(T, D), grid(V, D)
    h[:, 1 + 30:], w[:, 1 + 30:] = 0.0, 0.0  # (30 products of at most 1)
    h[:, 0], w[:, 0] = first, common
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    if T > 4:
        t[::7] = -1
    return h.to(DT[dtype]), w.to(DT[dtype]), t


def check(h, w, t, scale, g, gh, dtype):
    """The gradient after the forward call, against the definition in 64 bits with lse itself."""
    lp, H, lse = forward(h, w, t, scale)
    dh, dw = backward(h, w, t, scale, lse, H if gh is not None else None, g, gh)
    s = float(np.float32(scale))
    V, T = w.shape[0], len(t)
    x = h.double() @ w.double().t()  # (exact)
    z = s * (x - x.amax(1, keepdim=True))
    q = z - torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(q)
    ent = -(p * q.clamp_min(-1e6)).sum(1, keepdim=True)
    gg = torch.where(t >= 0, g, torch.zeros_like(g)).double()[:, None]
    hh = gh.double()[:, None] if gh is not None else torch.zeros_like(gg)
    inner = gg + hh * (q.clamp_min(-1e6) + ent)
    c = -p * inner
    c.scatter_add_(1, t.clamp_min(0)[:, None], gg)
    c *= s
    # of lp: its own rounding, those of a sum of V exponentials and its logarithm
    q = q.clamp_min(-200.0)
    dz = U * (4 * q.abs() + 32 + 4 * math.sqrt(V))
    e = s * p * (inner.abs() * dz + 2 * U * gg.abs()
                 + hh.abs() * (dz + 2 * U * (ent + q.abs() + 4 * ent * math.sqrt(V))))
    low = 2 * s * (gg.abs() + 4 * hh.abs()).max() * 2.0 ** -39 if dtype == "f16" else 0.0
    e = e + EPS[dtype] * (c.abs() + e) + low + TINY["bf16"]
    for got, want, tol in (
            (dh, c @ w.double(), (e + STEP * V * c.abs()) @ w.double().abs()),
            (dw, c.t() @ h.double(), (e + STEP * T * c.abs()).t() @ h.double().abs())):
        tol = tol + EPS[dtype] * (want.abs() + tol) + TINY[dtype]
        assert not got.isnan().any()
        bad = (got.double() - want).abs() > tol
        assert not bad.any(), (got[bad][:4], want[bad][:4], tol[bad][:4])


def gradients(T, ent):
    gen = torch.Generator(device="cuda").manual_seed(T)
    g = torch.randn((T,), generator=gen, device="cuda") / T
    return g, 0.1 * torch.randn((T,), generator=gen, device="cuda") / T if ent else None


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,D", [(1, 300, 32), (20, 1000, 64), (40, 700, 40), (130, 2000, 64),
                                   (300, 1025, 64), (600, 513, 32)])
@pytest.mark.parametrize("scale", [1.0, 1.0 / 0.7])
@pytest.mark.parametrize("first", [2.0 ** 9, -2.0 ** 9, 2.0 ** 6, -2.0 ** 5])
def test_gradient_of_far_logits(dtype, T, V, D, scale, first):
    """Logits around 2^17, -2^17, 2^14 and -2^13."""
    h, w, t = far_inputs(T, V, D, dtype, first, 2.0 ** 8)
    check(h, w, t, scale, *gradients(T, (T + V) % 3 != 0), dtype)


@pytest.mark.parametrize("T", [20, 300])
def test_near_and_far_positions_beside_each_other(T):
    """Positions on both sides of the size from which the row is summed again, masked ones among
    them."""
    h, w, t = far_inputs(T, 900, 48, "f16", 0.0, 2.0 ** 8)
    h[::3, 0], h[1::3, 0] = 512.0, 4.0
    check(h, w, t, 1.0 / 0.7, *gradients(T, True), "f16")


@pytest.mark.parametrize("T", [5, 77, 700])
@pytest.mark.parametrize("dtype,first,common", [
    ("f16", 2.0 ** 15, 2.0 ** 15), ("f16", -2.0 ** 15, 2.0 ** 15),
    ("bf16", 2.0 ** 40, 2.0 ** 40), ("bf16", -2.0 ** 63, 2.0 ** 63)])
def test_gradient_of_one_token_and_of_equal_ones(T, dtype, first, common):
    """Logits of 2^30, 2^80 and 2^126: all equal, and of one token that holds all mass."""
    V, D, scale = 600, 16, 1.0 / 0.7
    h = torch.zeros((T, D), dtype=DT[dtype], device="cuda")
    w = torch.zeros((V, D), dtype=DT[dtype], device="cuda")
    h[:, 0], w[:, 0] = first, common
    h[:, 1] = 1.0
    t = torch.arange(T, device="cuda") % V
    check(h, w, t, scale, *gradients(T, True), dtype)
    w[9, 0] = common * (1.25 if first > 0 else 0.75)
    t[::2] = 9
    check(h, w, t, scale, *gradients(T, True), dtype)


def test_far_positions_of_several_passes():
    """More positions than one pass of the sums takes, in several pieces of the vocabulary."""
    T, V, D = 16500, 8300, 32
    h, w, t = far_inputs(T, V, D, "bf16", 2.0 ** 9, 2.0 ** 8)
    h[::2, 0] = 1.0
    check(h, w, t, 1.25, *gradients(T, True), "bf16")


def test_far_gradient_captured_and_replayed():
    """One graph serves near states and far ones: what a call needs is decided on the device."""
    T, V, D = 300, 900, 48
    h, w, t = far_inputs(T, V, D, "bf16", 0.0, 2.0 ** 8)
    g, gh = gradients(T, True)
    lp, H, lse = (torch.zeros((T,), device="cuda") for _ in range(3))
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    ws = torch.empty((max(bt.boute_hidden_logprobs_workspace(h, w, b) for b in (False, True)),),
                     dtype=torch.uint8, device="cuda")

    def step():
        bt.boute_hidden_logprobs(h, w, t, 1.25, lp, H, lse, ws)
        bt.boute_hidden_logprobs_grad(h, w, t, 1.25, lse, H, g, gh, dh, dw, ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for first in (512.0, 0.0, -512.0):
            h[:, 0] = first
            graph.replay()
            s.synchronize()
            l2, H2, lse2 = forward(h, w, t, 1.25)
            want = backward(h, w, t, 1.25, lse2, H2, g, gh)
            assert torch.equal(dh, want[0]) and torch.equal(dw, want[1])
    check(h, w, t, 1.25, g, gh, "bf16")
