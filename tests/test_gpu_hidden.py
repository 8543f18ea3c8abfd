"""Log-probabilities from hidden states and the vocabulary's weight, and their gradient, against
plain forms in 64 bits: sizes around the tiles, odd ones, pitches and addresses, targets that are
none, masked, infinite and NaN rows, several pieces and passes, streams and graphs.

Tolerances. A logit is a sum of D products that fp32 holds exactly, 16 a step: a step aligns them and
the sum so far to the largest of the 17 and may lose a unit of each, 2^-24 = U relative to the
largest, which is A = sum |h w| at most: 17/16 D U A in all. The softmax adds what the
log-probabilities of given logits have: U (8 (2 + spread) + 4 sqrt(V)), for lse 2 U |lse| more, for
the entropy, whose terms are weighted with up to 2 + ln V, times that (twice for the logits' own
error). A gradient's coefficient has p's error (relative: the logit's and the exponent's roundings),
one rounding to the type (EPS; fp16 in scaled units whose smallest step is 2^-38 of the largest bound,
half of that rounded), and its products the sums' errors, 17/16 U a term over T or V terms."""
import math

import numpy as np
import pytest
import torch

from _answers import U
from paper_2602_10729_gb300 import boute as bt

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}
F32, I64 = torch.float32, torch.int64
STEP = 17 / 16 * U


def placed(x, pitch=0, shift=0):
    R, D = x.shape
    buf = torch.full((R * (D + pitch) + shift,), float("nan"), dtype=x.dtype, device="cuda")
    out = buf[shift:].view(R, D + pitch)[:, :D]
    out.copy_(x)
    return out


def inputs(T, V, D, dtype, pitch=0, shift=0, seed=0, spread=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000 + T + V + D)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    w = (randn(V, D) * (spread / math.sqrt(D))).to(DT[dtype])
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    h = (randn(T, D) + 3.0 * torch.rand((T, 1), generator=g, device="cuda") * w[t].float()).to(DT[dtype])
    if T > 4:
        t[torch.rand((T,), generator=g, device="cuda") < 0.1] = -1
    return placed(h, pitch, shift), placed(w, pitch, shift), t


def forward(h, w, t, scale, stream=None, ws=None):
    lp, H, lse = (torch.full((h.shape[0],), 9.0, device="cuda") for _ in range(3))
    n = bt.boute_hidden_logprobs_workspace(h, w)
    if ws is None:
        ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    bt.boute_hidden_logprobs(h, w, t, scale, lp, H, lse, ws, stream)
    return lp, H, lse


def backward(h, w, t, scale, lse, H, g, gh, pitch=0, shift=0, stream=None):
    dh, dw = (placed(torch.zeros_like(x) + 5.0, pitch, shift) for x in (h, w))
    n = bt.boute_hidden_logprobs_workspace(h, w, True)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    bt.boute_hidden_logprobs_grad(h, w, t, scale, lse, H, g, gh, dh, dw, ws, stream)
    return dh, dw


class Plain:
    """In 64 bits, in pieces of the positions."""

    def __init__(self, h, w, t, scale):
        self.h, self.w, self.t = h.double(), w.double(), t
        self.scale = float(np.float32(scale))
        V, D = w.shape
        lp, H, lse, dz = [], [], [], []
        for r in self.parts():
            z, size = self.logits(r)
            e = STEP * D * size * self.scale  # of a logit
            m = torch.logsumexp(z, 1)
            q = z - m[:, None]
            p = torch.exp(q)
            H.append(-(p * q.clamp_min(-1e6)).sum(1))
            lp.append(torch.where(t[r] >= 0, q.gather(1, t[r].clamp(0, V - 1)[:, None])[:, 0],
                                  torch.zeros_like(m)))
            lse.append(m)
            spread = (z.amax(1) - z.amin(1)).clamp(max=200.0)
            dz.append(e.amax(1) + U * (8 * (2 + spread) + 4 * math.sqrt(V)))
        self.lp, self.H, self.lse, self.tol = (torch.cat(x) for x in (lp, H, lse, dz))

    def parts(self):
        n = max(1, min(512, (1 << 26) // self.w.shape[0]))
        return [slice(r, min(r + n, len(self.t))) for r in range(0, len(self.t), n)]

    def logits(self, r):
        return self.scale * (self.h[r] @ self.w.t()), self.h[r].abs() @ self.w.t().abs()

    def check(self, lp, H, lse):
        V = self.w.shape[0]
        assert ((lse.double() - self.lse).abs() <= self.tol + 2 * U * self.lse.abs()).all()
        tol = 2 * self.tol + 2 * U * self.lp.abs()
        assert ((lp.double() - self.lp).abs() <= tol).all()
        assert (lp[self.t < 0] == 0).all()
        tol = 2 * self.tol * (2 + math.log(V)) + 2 * U * self.H
        assert ((H.double() - self.H).abs() <= tol).all()

    def grad(self, g, gh, dtype, coef=None):
        """(dh, dw, their tolerances) of the outputs' gradients, with lse and the entropy rounded to fp32;
        coef: the relative error of a coefficient's rounding."""
        coef = EPS[dtype] if coef is None else coef
        V, D = self.w.shape
        T = len(self.t)
        g = torch.where(self.t >= 0, g, torch.zeros_like(g)).double()
        gh = gh.double() if gh is not None else torch.zeros_like(g)
        dw, tw = torch.zeros_like(self.w), torch.zeros_like(self.w)
        dh, th = [], []
        most = self.scale * (g.abs() + 4 * gh.abs()).max().item()
        low = 2 * most * 2.0 ** -39 if dtype == "f16" else 0.0
        lse, H = self.lse.float().double(), self.H.float().double()
        for r in self.parts():
            z, size = self.logits(r)
            q = z - lse[r, None]
            p = torch.exp(q)
            inner = g[r, None] + gh[r, None] * (q + H[r, None])
            c = -p * inner
            at = (self.t[r] >= 0).nonzero()[:, 0]
            c[at, self.t[r][at]] += g[r][at]
            c *= self.scale
            dz = STEP * D * size * self.scale + U * (4 * q.abs() + 4 * lse[r, None].abs() + 16)
            e = self.scale * p * ((inner.abs() + 2 * U * (g[r].abs() + gh[r].abs() * (H[r] + 1))[:, None])
                                  * dz + gh[r, None].abs() * (dz + 2 * U * (H[r, None] + q.abs())))
            e += coef * (c.abs() + e) + low + TINY["bf16"]
            dh.append(c @ self.w)
            th.append((e + STEP * V * c.abs()) @ self.w.abs())
            dw += c.t() @ self.h[r]
            tw += (e + STEP * T * c.abs()).t() @ self.h[r].abs()
        dh, th = torch.cat(dh), torch.cat(th)
        end = lambda x, e: e + EPS[dtype] * (x.abs() + e) + TINY[dtype]
        return dh, dw, end(dh, th), end(dw, tw)


SIZES = [  # T, V, D, dtype, scale, pitch, shift
    (1, 1, 1, "bf16", 1.0, 0, 0), (1, 2, 8, "f16", 1.0, 0, 0), (2, 31, 16, "bf16", 0.5, 0, 0),
    (5, 300, 64, "f16", 1.25, 0, 0), (32, 256, 64, "bf16", 1.0, 0, 0),
    (33, 257, 72, "bf16", 1.0 / 0.7, 8, 0), (64, 512, 128, "f16", 1.0, 0, 8),
    (65, 511, 200, "bf16", 1.0, 24, 16), (255, 1000, 128, "bf16", 1.0, 0, 0),
    (256, 1024, 64, "f16", 1.0, 0, 0), (257, 1025, 136, "f16", 1.25, 0, 0),
    (300, 1001, 1001, "bf16", 1.0, 0, 0), (100, 700, 520, "f16", 1.0, 0, 3),
    (77, 900, 63, "bf16", 1.0, 1, 1), (515, 5000, 1000, "f16", 1.0 / 0.7, 0, 0),
    (600, 777, 4096, "bf16", 1.0, 0, 0), (1, 50021, 2048, "bf16", 1.0, 0, 0),
    (1, 3000, 515, "f16", 1.0, 0, 1), (700, 40000, 32, "bf16", 1.0, 0, 0)]


@pytest.mark.parametrize("T,V,D,dtype,scale,pitch,shift", SIZES)
def test_forward(T, V, D, dtype, scale, pitch, shift):
    h, w, t = inputs(T, V, D, dtype, pitch, shift)
    got = forward(h, w, t, scale)
    Plain(h, w, t, scale).check(*got)
    assert all(torch.equal(a, b) for a, b in zip(got, forward(h, w, t, scale)))


def check_grad(T, V, D, dtype, scale, pitch=0, shift=0, ent=True, spread=1.5):
    h, w, t = inputs(T, V, D, dtype, pitch, shift, seed=1, spread=spread)
    gen = torch.Generator(device="cuda").manual_seed(T + D)
    g = torch.randn((T,), generator=gen, device="cuda") / T
    gh = 0.1 * torch.randn((T,), generator=gen, device="cuda") / T if ent else None
    plain = Plain(h, w, t, scale)
    lse, H = plain.lse.float(), plain.H.float()
    got = backward(h, w, t, scale, lse, H if ent else None, g, gh, pitch, shift)
    dh, dw, th, tw = plain.grad(g, gh, dtype)
    assert ((got[0].double() - dh).abs() <= th).all()
    assert ((got[1].double() - dw).abs() <= tw).all()
    again = backward(h, w, t, scale, lse, H if ent else None, g, gh, pitch, shift)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("T,V,D,dtype,scale,pitch,shift", SIZES)
def test_gradient(T, V, D, dtype, scale, pitch, shift):
    check_grad(T, V, D, dtype, scale, pitch, shift, ent=(T + V) % 3 != 0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 5, 31, 32])
def test_gradients_of_few_positions_keep_the_coefficients_low_parts(T, dtype):
    """Up to 32 positions: a coefficient is two numbers of the type, and off by EPS^2 alone."""
    h, w, t = inputs(T, 1000, 72, dtype, seed=4, spread=0.5)
    gen = torch.Generator(device="cuda").manual_seed(T)
    g, gh = (torch.randn((T,), generator=gen, device="cuda") for _ in range(2))
    plain = Plain(h, w, t, 1.0)
    got = backward(h, w, t, 1.0, plain.lse.float(), plain.H.float(), g, gh)
    dh, dw, th, tw = plain.grad(g, gh, dtype, EPS[dtype] ** 2)
    assert ((got[0].double() - dh).abs() <= th).all()
    assert ((got[1].double() - dw).abs() <= tw).all()


@pytest.mark.parametrize("T", [8191, 8192, 8193, 8200, 16500])
def test_positions_of_several_passes(T):
    h, w, t = inputs(T, 600, 64, "bf16")
    Plain(h, w, t, 1.0).check(*forward(h, w, t, 1.0))


@pytest.mark.parametrize("V", [16448, 20000])
def test_gradient_in_several_pieces_of_the_vocabulary(V):
    """8192 positions: pieces of 16384 tokens; the last is shorter than dh's parts with 16448."""
    check_grad(8192, V, 32, "bf16", 1.0)


def test_targets_beyond_the_vocabulary_and_none():
    h, w, t = inputs(40, 500, 64, "bf16")
    t = t.clone()
    t[0], t[1], t[2], t[3], t[4] = 500, 1 << 40, -1, -(1 << 50), 499
    lp, H, lse = forward(h, w, t, 1.0)
    assert lp[:2].isnan().all() and (lp[2:4] == 0).all() and not lp[4:].isnan().any()
    assert not (H.isnan() | lse.isnan()).any()
    g = torch.ones((40,), device="cuda")
    dh, dw = backward(h, w, t, 1.0, lse, H, g, g)
    assert dh[:2].isnan().all() and not dh[2:].isnan().any() and dw.isnan().all()
    keep = torch.arange(40, device="cuda") > 1
    dh, dw = backward(h[keep], w, t[keep], 1.0, lse[keep], H[keep], g[keep], None)
    assert not (dh.isnan().any() or dw.isnan().any())
    assert (dh[:2] == 0).all()  # (no token, and no gradient of the entropy)


def test_infinite_and_nan_rows():
    """A NaN or +inf logit leaves its position without a distribution; -inf masks a token; a position
    without a token left has lse -inf and entropy 0, and gradient 0."""
    T, V, D = 40, 600, 64
    h, w, t = inputs(T, V, D, "bf16")
    h, w, t = h.clone(), w.clone(), t.clone()
    h[:, 0], w[:, 0] = 0.0, 0.0
    h[:, 1], w[:, 1] = 0.0, 1.0
    w[7, 0] = -float("inf")  # times h[t, 0]
    h[:, 0] = 1.0            # token 7 is masked in every position
    h[3, 5] = float("nan")
    h[5, 0] = -1.0           # token 7 at +inf
    h[8, 1] = -float("inf")  # all masked
    t[1], t[2], t[8], t[9] = 7, 3, 4, -1
    lp, H, lse = forward(h, w, t, 1.0)
    for bad in (3, 5):
        assert lse[bad].isnan() and H[bad].isnan()
    assert lse[8] == -float("inf") and H[8] == 0 and lp[8] == -float("inf")
    assert lp[1] == -float("inf") and lp[9] == 0
    fine = torch.ones(T, dtype=torch.bool, device="cuda")
    fine[[3, 5, 8]] = False
    rest = torch.arange(V, device="cuda") != 7
    t2 = torch.where(t > 7, t - 1, t)
    ok = fine & (t != 7)
    hh = h.clone()
    hh[:, 0] = 0.0
    Plain(hh[ok], w[rest].clone().nan_to_num(0.0), t2[ok], 1.0).check(lp[ok], H[ok], lse[ok])
    g = torch.full((T,), 0.5, device="cuda")
    dh, dw = backward(h[fine], w, t[fine], 1.0, lse[fine], H[fine], g[fine], g[fine])
    assert not dh[:, 2:].isnan().any() and not dw[:, 2:].isnan().any()
    dh, _ = backward(h, w, t, 1.0, lse, H, g, g)
    assert dh[3].isnan().all() and dh[5].isnan().all()


def test_a_scale_that_overflows():
    """z = scale x beyond fp32: +inf leaves no distribution, -inf masks; what stays finite counts."""
    V, D = 300, 16
    h = torch.zeros((3, D), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    h[0, 0], h[1, 1], h[2, 2] = 1.0, 1.0, 1.0
    w[5, 0] = 2.0 ** 40            # position 0: one logit to +inf
    w[:, 1] = -2.0 ** 40           # position 1: all to -inf
    w[:, 2], w[7, 2] = -2.0 ** 40, 2.0 ** -90  # position 2: all but token 7
    t = torch.tensor([0, 3, 7], device="cuda")
    lp, H, lse = forward(h, w, t, 2.0 ** 100)
    assert lp[0].isnan() and H[0].isnan() and lse[0].isnan()
    assert lse[1] == -float("inf") and H[1] == 0 and lp[1] == -float("inf")
    assert lse[2] == 2.0 ** 10 and H[2] == 0 and lp[2] == 0


def test_a_position_without_a_token_left_has_gradient_0():
    T, V, D = 33, 300, 40
    h, w, t = inputs(T, V, D, "f16")
    lp, H, lse = forward(h, w, t, 1.0)
    lse[4], H[4] = -float("inf"), 0.0
    g = torch.ones((T,), device="cuda")
    dh, dw = backward(h, w, t, 1.0, lse, H, g, g)
    assert (dh[4] == 0).all() and not dw.isnan().any()
    keep = torch.arange(T, device="cuda") != 4
    _, want = backward(h[keep], w, t[keep], 1.0, lse[keep], H[keep], g[keep], g[keep])
    # (the same sums but for their steps' grouping)
    assert ((dw.double() - want.double()).abs() <= 4 * EPS["f16"] * want.double().abs() + 1e-3).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", [1e-30, 1e-8, 1.0, 1e6])
def test_gradients_of_any_size(dtype, size):
    """The coefficients are scaled while they have 16 bits: what the outputs' types hold is as good."""
    T, V, D = 130, 700, 96
    h, w, t = inputs(T, V, D, dtype)
    plain = Plain(h, w, t, 1.0)
    g = torch.randn((T,), device="cuda") * size
    got = backward(h, w, t, 1.0, plain.lse.float(), plain.H.float(), g, None)
    dh, dw, th, tw = plain.grad(g, None, dtype)
    lim = 65504.0 if dtype == "f16" else 3e38
    for a, b, e in ((got[0], dh, th), (got[1], dw, tw)):
        ok = b.abs() + e < lim
        assert ok.any() and ((a.double() - b).abs() <= e)[ok].all()


def test_gradient_0():
    h, w, t = inputs(50, 400, 48, "f16")
    lp, H, lse = forward(h, w, t, 1.0)
    z = torch.zeros((50,), device="cuda")
    dh, dw = backward(h, w, t, 1.0, lse, H, z, z)
    assert not dh.any() and not dw.any()


def test_without_positions():
    h = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.randn((300, 64), device="cuda").bfloat16()
    e = torch.empty((0,), device="cuda")
    t = torch.empty((0,), dtype=I64, device="cuda")
    ws = torch.empty((bt.boute_hidden_logprobs_workspace(h, w, True) + 256,), dtype=torch.uint8,
                     device="cuda")
    bt.boute_hidden_logprobs(h, w, t, 1.0, e, e, e, ws)
    dw = torch.full((300, 70), 5.0, dtype=torch.bfloat16, device="cuda")
    bt.boute_hidden_logprobs_grad(h, w, t, 1.0, e, None, e, None, torch.empty_like(h), dw[:, :64], ws)
    assert not dw[:, :64].any() and (dw[:, 64:] == 5).all()


def test_gradient_against_differences():
    """The slope of f = <u, logprob> + <v, entropy> along a direction, from the forward call in fp32 at
    steps of h that 16 bits hold, against <dh, direction> (and the same for w)."""
    T, V, D, eps = 24, 300, 32, 2.0 ** -5
    g = torch.Generator(device="cuda").manual_seed(11)
    grid = lambda *s: (torch.randint(-16, 17, s, generator=g, device="cuda") / 16.0).half()
    h, w, t = grid(T, D), grid(V, D), torch.randint(0, V, (T,), generator=g, device="cuda")
    u, v = torch.randn((T,), generator=g, device="cuda"), torch.randn((T,), generator=g, device="cuda")
    lp, H, lse = forward(h, w, t, 1.0)
    dh, dw = backward(h, w, t, 1.0, lse, H, u, v)

    def f(h, w):
        lp, H, _ = forward(h, w, t, 1.0)
        return (u.double() * lp.double() + v.double() * H.double())

    for x, dx in ((h, dh), (w, dw)):
        d = torch.randint(-1, 2, x.shape, generator=g, device="cuda").half()
        a = lambda s: (x.double() + s * eps * d.double()).half()  # (exact: sixteenths and 32nds)
        at = lambda s: f(a(s), w) if x is h else f(h, a(s))
        want = (dx.double() * d.double()).sum()
        slope = (8 * (at(1) - at(-1)) - (at(2) - at(-2))).sum() / (12 * eps)
        # the five-point formula leaves eps^4 f'''''/30 (logits move by 32 * 1 * eps at most along d:
        # a random walk of some 5 eps), the forward call's roundings 1e-6 / eps a position, and the
        # gradient EPS of the sums of its magnitudes
        tol = (T * (5 ** 5) * eps ** 4 * 3 / 30 + T * 1e-5 / eps * 2
               + 4 * EPS["f16"] * (dx.double().abs() * d.double().abs()).sum())
        assert (slope - want).abs() <= tol, (slope, want, tol)


def test_against_the_call_that_takes_logits():
    """Its outputs and its gradient, for the logits that torch makes of the same states."""
    T, V, D = 130, 2000, 256
    h, w, t = inputs(T, V, D, "bf16")
    lp, H, lse = forward(h, w, t, 1.25)
    x = (h.double() @ w.double().t()).float()
    a, b, c = (torch.empty((T,), device="cuda") for _ in range(3))
    bt.boute_token_logprobs(x, t, 1.25, a, b, c)
    tol = Plain(h, w, t, 1.25).tol
    assert ((lp - a).abs() <= 4 * tol).all() and ((lse - c).abs() <= 4 * tol).all()
    assert ((H - b).abs() <= 4 * tol * (2 + math.log(V))).all()


def test_a_run_to_answers_scores_and_back_in_a_graph():
    """hidden states -> log-probabilities -> answers' scores and back, captured on a stream of its own
    and replayed with other states; the same workspace serves both calls, one after another."""
    T, V, D, Q = 300, 3000, 128, 7
    h, w, t = inputs(T, V, D, "bf16")
    off = torch.tensor([0, 40, 40, 100, 180, 181, 260, 300], dtype=I64, device="cuda")
    new = lambda *s: torch.zeros(s, device="cuda")
    lp, H, lse, gl, gh = (new(T) for _ in range(5))
    scores, counts = new(Q, 4), torch.zeros((Q,), dtype=torch.int32, device="cuda")
    gs = torch.randn((Q, 4), device="cuda")
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    ws = torch.empty((max(bt.boute_hidden_logprobs_workspace(h, w, b) for b in (False, True)),),
                     dtype=torch.uint8, device="cuda")

    def step():
        bt.boute_hidden_logprobs(h, w, t, 1.0, lp, H, lse, ws)
        bt.boute_answer_scores(lp, H, t, off, scores, counts)
        bt.boute_answer_scores_grad(lp, H, t, off, gs, gl, gh)
        bt.boute_hidden_logprobs_grad(h, w, t, 1.0, lse, H, gl, gh, dh, dw, ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        h2, _, _ = inputs(T, V, D, "bf16", seed=5)
        h.copy_(h2)
        graph.replay()
    s.synchronize()
    Plain(h, w, t, 1.0).check(lp, H, lse)
    got = [x.clone() for x in (dh, dw, scores)]
    step()
    assert all(torch.equal(a, b) for a, b in zip(got, (dh, dw, scores)))
    on = (t[:40] >= 0)
    assert (scores[0, 0].double() - lp[:40][on].double().mean()).abs() < 1e-5
    plain = Plain(h, w, t, 1.0)
    plain.lse, plain.H = lse.double(), H.double()
    a, b, ta, tb = plain.grad(gl, gh, "bf16")
    assert ((dh.double() - a).abs() <= ta).all() and ((dw.double() - b).abs() <= tb).all()


def test_two_calls_at_once_on_streams_of_their_own():
    sets = [inputs(200, 4000, 256, "bf16", seed=i) for i in range(2)]
    alone = [forward(*s, 1.0) for s in sets]
    ws = [torch.empty((bt.boute_hidden_logprobs_workspace(*s[:2]),), dtype=torch.uint8, device="cuda")
          for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        out = []
        for s, st, m in zip(sets, streams, ws):
            with torch.cuda.stream(st):
                out.append(forward(*s, 1.0, ws=m))
        torch.cuda.synchronize()
        for a, b in zip(out, alone):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_rows_beyond_the_arrays_are_left_as_they_were():
    h, w, t = inputs(37, 333, 56, "f16", pitch=8)
    plain = Plain(h, w, t, 1.0)
    bufs = [torch.full((x.shape[0] + 2, 64), 5.0, dtype=x.dtype, device="cuda") for x in (h, w)]
    outs = [b[1:-1, :56] for b in bufs]
    g = torch.ones((37,), device="cuda")
    ws = torch.empty((bt.boute_hidden_logprobs_workspace(h, w, True),), dtype=torch.uint8, device="cuda")
    bt.boute_hidden_logprobs_grad(h, w, t, 1.0, plain.lse.float(), None, g, None, *outs, ws)
    for b in bufs:
        assert (b[0] == 5).all() and (b[-1] == 5).all() and (b[:, 56:] == 5).all()
        assert not (b[1:-1, :56] == 5).all(1).any()
