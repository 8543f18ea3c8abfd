"""What long sums lose on the way to log-probabilities from hidden states and their gradient. The
tensor cores cut off what fp32 does not hold beside the sum so far, 16 terms a step, up to a unit,
2 U = 2^-23, each: sums are taken in parts, so that many steps do not add up to a bias."""
import math

import pytest
import torch

from test_gpu_hidden import DT, EPS, U, backward, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,dtype", [
    (5000, "f16"), (16384, "f16"), (16385, "f16"), (40000, "f16"), (131072, "f16"), (1 << 20, "f16"),
    (5000, "bf16"), (131072, "bf16"), (131073, "bf16"), (1 << 20, "bf16")])
def test_the_weights_gradient_of_many_positions(T, dtype):
    """Each element is a sum over the positions of terms of one sign. Its relative error, averaged over
    the elements, is the bias of the sum: the roundings to 16 bits, of the coefficients and of the result,
    are apart by element or position. Up to 256 x 64 positions (bf16: 2048 x 64) a sum has a step for 16 of
    them, beyond that parts of 64 x 64 have 256; a step loses 2 U at most. p's own errors are 2 ulp of an exponential
    and lse's rounding (lse < 8)."""
    V, D = 300, 40
    g = torch.Generator(device="cuda").manual_seed(T)
    by = 1 + torch.rand((D,), generator=g, device="cuda")  # (sums apart, and with them their roundings)
    h = (by + 0.25 * torch.rand((T, D), generator=g, device="cuda")).to(DT[dtype])
    w = (0.1 * torch.randn((V, D), generator=g, device="cuda")).to(DT[dtype])
    t = torch.full((T,), 7, dtype=torch.int64, device="cuda")
    up = torch.rand((T,), generator=g, device="cuda") / T
    lp, H, lse = forward(h, w, t, 1.0)
    _, dw = backward(h, w, t, 1.0, lse, None, up, None)
    want = torch.zeros((V, D), dtype=torch.float64, device="cuda")
    for r in range(0, T, 1 << 16):
        x = h[r:r + (1 << 16)].double()
        c = -torch.softmax(x @ w.double().t(), 1)
        c[:, 7] += 1
        want += (c * up[r:r + (1 << 16), None].double()).t() @ x
    error = (dw.double() - want) / want
    # six deviations of the mean: the result's rounding (within EPS, uniform) and, by token, the
    # coefficients'; and what elements below fp16's normal range lose
    noise = 6 * EPS[dtype] / math.sqrt(3) * (1 / math.sqrt(V * D) + 1 / math.sqrt(V * T / 2))
    least = 2.0 ** -25 if dtype == "f16" else 0.0
    tiny = (least / want.abs()).mean().item() * 6 / math.sqrt(V * D)
    steps = T / 16 if T <= (16384 if dtype == "f16" else 131072) else 256
    assert abs(error.mean().item()) <= steps * 2 * U + 16 * U + noise + tiny
    assert (error.abs() <= 2 * EPS[dtype] + least / want.abs()).all()


@pytest.mark.parametrize("T", [3, 40, 130, 300, 600])
@pytest.mark.parametrize("D", [2048, 4096])
def test_gradient_of_logits_with_a_large_common_term(T, D):
    """Each logit begins with 512, beside which fp32 holds multiples of 2^-14: 32 steps, which a part of
    512 elements has, are off by 32 units at most and by their random half, 2^-14 sqrt(32 / 12), from
    one token to another (of 16 blocks, sqrt(64 / 12)); all steps of 4096 elements were off by 255 2^-15
    throughout. The entropy's gradient, whose coefficients p (ln p + H) show it, is otherwise off by its
    roundings to 16 bits: EPS relative, and 2^-25 at least, as many of dw's elements are below 2^-14,
    where fp16 has no finer step than 2^-24 (600 positions: elements of 9e-6, of which 2^-25 / sqrt(3),
    uniform, is 2e-3)."""
    V = 2000
    h, w, t = inputs(T, V, D, "f16", seed=3)
    h[:, :16], w[:, :16] = 0, 0
    h[:, 0], w[:, 0] = 16.0, 32.0
    gh = torch.randn((T,), device="cuda") / T
    lp, H, lse = forward(h, w, t, 1.0)
    dh, dw = backward(h, w, t, 1.0, lse, H, torch.zeros_like(gh), gh)
    q = torch.log_softmax(h.double() @ w.double().t(), 1)
    c = -gh.double()[:, None] * q.exp() * (q - (q.exp() * q).sum(1, keepdim=True))
    p = 2.0 ** -14 * math.sqrt(64 / 12) + U * 512  # of ln p: in p, and beside 1 or so in ln p + H
    tol = 2 * p + 2 * EPS["f16"] / math.sqrt(3)
    for got, want in ((dh, c @ w.double()), (dw, c.t() @ h.double())):
        got, want = got.double()[:, 16:], want[:, 16:]
        least = 2.0 ** -25 / math.sqrt(3) * math.sqrt(want.numel())
        assert (got - want).norm() <= tol * want.norm() + least, (got - want).norm() / want.norm()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,D", [(3, 700), (20, 1100), (64, 2048), (130, 1100), (300, 2048), (600, 1500)])
def test_far_positions_coefficients_sum_to_0(T, D, dtype):
    """Logits around 2^17, whose sums fp32 rounds to multiples of 2^-7 in an order of their own: the
    coefficients' are those of which the largest and ln s were taken, so that p sums to 1. One element
    of all tokens is 1 and adds a position's coefficients up: what they leave is their rounding (EPS
    each; of the target's and of the others' together, g scale each) and that of p's sum."""
    h, w, t = inputs(T, 1500, D, dtype, seed=8)
    h[:, 0], w[:, 0] = 2.0 ** 9, 2.0 ** 8
    h[:, -1], w[:, -1] = 0.0, 1.0
    t = t.clamp_min(0)
    g = torch.rand((T,), device="cuda") + 0.5
    lp, H, lse = forward(h, w, t, 1.25)
    assert (lse > 1e5).all()
    dh, _ = backward(h, w, t, 1.25, lse, None, g, None)
    tol = 1.25 * g.double() * (2 * EPS[dtype] + 64 * U)
    assert (dh[:, -1].double().abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [60, 130, 600, 3000])
@pytest.mark.parametrize("D", [512, 1024, 2048, 4096, 16384])
def test_how_far_the_outputs_are_off(T, D, dtype):
    """Relative 2-norms, at twice what is documented beside the parts: 2e-7 in parts of 512 elements, which
    up to 64 positions and reductions of more than 2048 elements have, 4e-7 in others."""
    h, w, t = inputs(T, 5000, D, dtype, seed=9)
    lp, H, lse = forward(h, w, t, 1.0)
    for r in range(0, T, 1000):
        r = slice(r, r + 1000)
        q = torch.log_softmax(h[r].double() @ w.double().t(), 1)
        m = torch.logsumexp(h[r].double() @ w.double().t(), 1)
        at = torch.where(t[r] >= 0, q.gather(1, t[r].clamp_min(0)[:, None])[:, 0], torch.zeros_like(m))
        tol = 4e-7 if T <= 64 or D > 2048 or D <= 512 else 8e-7
        for got, want in ((lp[r], at), (H[r], -(q.exp() * q).sum(1)), (lse[r], m)):
            assert (got.double() - want).norm() <= tol * want.norm()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [1, 20, 32, 33, 130, 600, 3000])
@pytest.mark.parametrize("D", [512, 4096])
def test_how_far_the_gradients_are_off(T, D, dtype):
    """Relative 2-norms: one rounding to the type is EPS / sqrt(3) at most, its relative size being uniform
    within EPS where a binade begins and half of that where it ends. Up to 32 positions that is all, with
    more the coefficients' is there too, apart from the result's. (A tenth beyond: some hundred elements
    at least, and logits' errors of 1e-6.)"""
    h, w, t = inputs(T, 3000, D, dtype, seed=10)
    g, gh = torch.randn((T,), device="cuda"), 0.3 * torch.randn((T,), device="cuda")
    lp, H, lse = forward(h, w, t, 1.0)
    dh, dw = backward(h, w, t, 1.0, lse, H, g, gh)
    q = torch.log_softmax(h.double() @ w.double().t(), 1)
    c = -q.exp() * (torch.where(t >= 0, g, 0 * g).double()[:, None]
                    + gh.double()[:, None] * (q - (q.exp() * q).sum(1, keepdim=True)))
    at = (t >= 0).nonzero()[:, 0]
    c[at, t[at]] += g[at].double()
    tol = 1.1 * EPS[dtype] / math.sqrt(3) * (1 if T <= 32 else math.sqrt(2))
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0  # (half of fp16's smallest step)
    for got, want in ((dh, c @ w.double()), (dw, c.t() @ h.double())):
        assert (got.double() - want).norm() <= tol * want.norm() + tiny * math.sqrt(want.numel() / 3)
