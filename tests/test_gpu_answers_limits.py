"""The operators over a model's answers where their inputs or launches are at a limit, against plain
64-bit forms."""
import os
import subprocess
import sys
import textwrap

import numpy as np
import pytest
import torch

from _answers import (U, answer_grad, answer_rows, route_grad_row, route_row, scores,
                      token_grad_row)
from paper_2602_10729_gb300 import boute as bt
from test_gpu_answers import (DT, EPS, answers, check_forward, close, forward, logits, placed,
                              scored)
from test_gpu_routing import SIG, SOFT, rel_tol, routed

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- blocks that end at once
def test_clusters_of_empty_answers():
    """A cluster per answer, most of which are empty: their blocks reach the exchange at once."""
    lengths = [0] * 60 + [250001] + [0, 1] * 20
    lp, ent, t, off = answers(77, lengths)
    want, cnt = answer_rows(lp.numpy(), ent.numpy(), t.numpy(), off.numpy())
    g = torch.randn((len(lengths), 4), generator=torch.Generator().manual_seed(6))
    wl, wh = answer_grad(lp.numpy(), ent.numpy(), t.numpy(), off.numpy(), g.double().numpy())
    tol = U * 8 * (4 + 4 * np.sqrt(np.maximum(cnt, 1)))[:, None]
    for _ in range(20):
        got, n = scored(lp, ent, t, off)
        assert n.tolist() == cnt.tolist()
        assert np.array_equal(got[:, [1, 3]], want[:, [1, 3]].astype(np.float32))
        close(got[:, [0, 2]], want[:, [0, 2]], tol)
        gl, gh = torch.full_like(lp, 9.0).cuda(), torch.full_like(lp, 9.0).cuda()
        bt.boute_answer_scores_grad(lp.cuda(), ent.cuda(), t.cuda(), off.cuda(), g.cuda(), gl, gh)
        close(gl.cpu().numpy(), wl, 4 * U * 10)
        close(gh.cpu().numpy(), wh, 4 * U * 10)


def test_clusters_on_streams_at_once():
    """Rows in clusters, on streams whose blocks share the SMs."""
    x, t = logits(31, 100, 40001, "bf16")
    xs, ts = x.cuda(), t.cuda()
    torch.cuda.synchronize()
    want = forward(xs, ts, 1.0, 9)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = []
    for i in range(24):
        with torch.cuda.stream(streams[i % 4]):
            outs.append(forward(xs, ts, 1.0, 9))
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(want, out))
    check_forward(x, t, 1.0, 9, want)


# ---------------------------------------------------------------- logits far from 0
# With |lse| over 1024 the gradient takes p from the row: x - max is exact where p is not 0, its
# product with the scale has one rounding of |z - m| <= 200, ln s a few of 2 + ln V. So
#   |dx_j - want| <= scale (|g| + |gh| 2 (2 + ln V + d)) exp(-d) U (8 (2 + 200) + 4 sqrt(V))
# holds whatever the size of the logits (d = m - z_j); with the entropy given as the forward call
# had it (its own tolerance above enters through g_entropy p H: another 8 U (2 + 200) (2 + ln V)).
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [0.7, 1 / 0.7, 1.0])
@pytest.mark.parametrize("T,V", [(5, 11), (5, 5003), (4, 70001), (1300, 2049)])  # one block and more
@pytest.mark.parametrize("ent", [True, False])
def test_gradient_of_logits_far_from_zero(dtype, scale, T, V, ent):
    base, t = logits(V, T, V, "f32", spread=1.0)
    x = base.to(DT[dtype])
    low = torch.finfo(DT[dtype]).min
    far = {"f32": -1e9, "f16": -6e4, "bf16": -1e9}[dtype]
    x[0] = low                                        # uniform
    x[1] = far
    x[2] = (base[2] * 3 + {"f32": 1e6, "f16": 3e4, "bf16": 1e4}[dtype]).to(DT[dtype])
    x[3] = low
    x[3, :3] = far / 4                                # three tokens left
    if scale > 1:                                     # (a scaled lowest value is -inf: masked)
        x[0] = far / 2
    t[:4] = torch.tensor([0, -1, V - 1, 2])
    gen = torch.Generator().manual_seed(V)
    g, gh = torch.randn(T, generator=gen), torch.randn(T, generator=gen) if ent else None
    xs, ts = x.cuda(), t.cuda()
    lp, H, lse, _, _ = forward(xs, ts, scale, 0)
    dx = torch.full_like(xs, 5.0)
    bt.boute_token_logprobs_grad(xs, ts, scale, lse, H if ent else None, g.cuda(),
                                 gh.cuda() if ent else None, dx)
    tiny = {"f32": 1e-38, "f16": 2.0 ** -25, "bf16": 1e-38}[dtype]
    got = dx[:5].float().cpu().numpy()
    for r in range(len(got)):
        row = x[r].float().numpy()
        gr, hr = float(g[r]), float(gh[r]) if ent else 0.0
        want = token_grad_row(row, scale, int(t[r]), gr, hr)
        z = row.astype(np.float64) * float(np.float32(scale))
        d = np.minimum(z.max() - z, 200.0)
        rel = U * (8 * (2 + 200.0) + 4 * np.sqrt(V))
        part = abs(gr) * (t[r] >= 0).item() + abs(hr) * 4 * (2 + np.log(V) + d)
        tol = scale * rel * part * np.exp(-d) + np.abs(want) * (EPS[dtype] + 8 * U) + tiny
        close(got[r], want, tol)
    bt.boute_token_logprobs_grad(xs, ts, scale, lse, H if ent else None, g.cuda(),
                                 gh.cuda() if ent else None, xs)  # in place
    assert torch.equal(xs, dx)


# ---------------------------------------------------------------- scores that fp32 hardly holds
# A score is at least 2^-149 or 0. Of a weight that is not renormalised |got - want| is at most a
# score's relative error (that of the other tests) and two units of 2^-149, times the factor. A
# renormalised weight has the relative error alone, whatever the size of its sum: it is a quotient,
# of which only parts below 2^-123 may be lost.
def tiny_queries(E, dtype):
    """Logits whose scores lie between 2^-148 and 2^-60 beside one of 0 (softmax) or without."""
    x = torch.full((9, E), -1e4)
    x[:, 0] = 0.0
    some = torch.linspace(-102.0, -84.0, 6)
    x[0, 2:8] = some
    x[1, 2:8] = some.flip(0) + 2.0
    x[2, 2:8] = -88.0
    x[3, 2:8] = -100.0
    x[4, 2:8] = torch.tensor([-42.0, -90.0, -60.0, -95.0, -41.0, -87.0])
    x[5, 2:8] = torch.tensor([-2.5, -90.0, -60.0, -95.0, -89.0, -87.0])
    x[6, 2:8] = -150.0                 # none of them held: weights 0
    x[7, 2:8] = torch.tensor([-150.0, -99.0, -150.0, -101.0, -150.0, -96.0])
    x[8, 2:8] = torch.tensor([1.0, -99.0, -2.0, -101.0, 0.5, -96.0])
    return x.to(DT[dtype])


def tiny_weights(x, bias, mode, k, renorm, factor, T=None, load=True):
    rows = torch.arange(T or len(x)) % len(x)
    idx, w, _ = routed(x[rows].cuda(), bias, mode, 1, 1, 1, k, renorm, factor, load=load)
    xs, b = x.float().numpy(), None if bias is None else bias.cpu().numpy()
    idx, w = idx.cpu().numpy(), w.cpu().numpy()
    for r in range(len(x)):
        wi, ww, _ = route_row(xs[r], b, mode, 1, 1, 1, k, renorm, factor)
        assert idx[r].tolist() == wi, r
        lost = 2.0 ** -123 if renorm else 2.0 ** -148
        close(w[r], ww, 2 * rel_tol(xs[r]) * np.abs(ww) + factor * lost)
    again = torch.as_tensor(w[:len(x)])[rows].numpy()
    assert np.array_equal(w.view(np.int32), again.view(np.int32))


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("factor", [2.5, 8.0, 1e30])
@pytest.mark.parametrize("E,T,load", [(12, None, True), (12, None, False), (12, 9000, True),
                                      (100, 9000, True), (250, 9000, True), (300, None, True),
                                      (600, None, True)])
def test_weights_of_scores_that_fp32_hardly_holds(mode, renorm, factor, E, T, load):
    """The bias chooses: six experts of tiny scores, in an order of its own."""
    bias = torch.zeros(E)
    bias[0] = -10.0
    bias[2:8] = torch.tensor([3.0, 8.0, 4.0, 7.0, 5.0, 6.0])
    for dtype in ("f32", "bf16"):
        for k in (2, 6):
            tiny_weights(tiny_queries(E, dtype), bias.cuda(), mode, k, renorm, factor, T, load)


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("E,T", [(12, None), (12, 9000), (64, 9000), (250, 9000), (300, None)])
def test_logistic_weights_far_below_zero(renorm, E, T):
    """Without a bias, 16-bit and 32-bit logits: all scores of a query are tiny."""
    x = tiny_queries(E, "f32")[[0, 1, 2, 3, 4, 5, 8]]  # (scores of 0 are compared as logits)
    x[:, 0] = -1e4
    x[:, 2:8] += torch.arange(6) * 0.5  # (no ties by bf16's rounding)
    for dtype in ("f32", "f16", "bf16"):
        for k in (1, 4, 6):
            tiny_weights(x.to(DT[dtype]), None, SIG, k, renorm, 8.0, T)


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("groups", [False, True])
@pytest.mark.parametrize("E,T,load", [(12, None, True), (12, None, False), (12, 9000, True),
                                      (100, 9000, True), (250, 9000, True), (300, None, True),
                                      (1000, None, True)])
def test_choice_among_scores_that_fp32_hardly_holds(mode, groups, E, T, load):
    """Tiny scores decide: beside a bias of 0 whose best expert is out of service, and as groups'
    sums of two. (They are some units of 2^-149 apart, or 0 and equal.)"""
    for dtype in ("f32", "bf16"):
        x = tiny_queries(E, dtype)
        if groups:
            bias, a = None, (E // (4 if E < 200 else 10 if E < 300 else 12 if E == 300 else 40), 1, 2, 4)
            if mode == SIG:
                x[:, 0] = -1e4
        else:
            bias, a = torch.zeros(E), (1, 1, 1, 6)
            bias[0] = -float("inf")
        rows = torch.arange(T or len(x)) % len(x)
        idx, _, _ = routed(x[rows].cuda(), None if bias is None else bias.cuda(), mode, *a, True, 1.0,
                           load=load)
        xs = x.float().numpy()
        want = [route_row(r, None if bias is None else bias.numpy(), mode, *a, True, 1.0)[0] for r in xs]
        assert idx[:len(x)].tolist() == want
        assert torch.equal(idx, idx[:len(x)][rows.cuda()])


# Of a gradient the error is that of the other tests: of the scores' relative error times the terms
# that they scale, which for weights with a sum are w (|g| + sum w |g|), whatever the sum's size.
def tiny_gradient(x, mode, idx, renorm, factor, seed, pitch=0, shift=0):
    T, k = idx.shape
    g = torch.randn((T, k), generator=torch.Generator().manual_seed(seed))
    xs = placed(x, pitch, shift)
    dx = torch.full(x.shape, 9.0, dtype=x.dtype, device="cuda")
    bt.boute_route_grad(xs, mode, renorm, factor, idx.cuda(), g.cuda(), dx)
    got, xf = dx.float().cpu().numpy(), x.float().numpy()
    name = {v: n for n, v in DT.items()}[x.dtype]
    for r in range(T):
        i = idx[r].tolist()
        want = route_grad_row(xf[r], mode, i, g[r].tolist(), renorm, factor)
        s = scores(xf[r], mode)
        on = [e for e in i if e >= 0]
        if mode == SOFT and renorm:  # the same with w = s / S, in which what 64 bits leave of S - S is 0
            w = s[on] / s[on].sum() if s[on].sum() > 0 else 0.0 * s[on]
            gs = factor * np.array([g[r, j] for j in range(k) if i[j] >= 0], np.float64)
            want = np.zeros(len(want))
            want[on] = w * (gs - (w * gs).sum())
        gm = float(g[r].abs().max()) * factor
        terms = np.zeros(len(xf[r]))
        terms[on] = 2 * gm * (s[on] / s[on].sum() if renorm and s[on].sum() > 0 else s[on])
        if mode == SOFT and not renorm:
            terms = gm * (terms > 0) * s + gm * s * s[on].sum()
        tiny = 2.0 ** -25 if name == "f16" else factor * 2.0 ** -122
        close(got[r], want, 4 * rel_tol(xf[r]) * terms + np.abs(want) * EPS[name] * 1.01 + tiny)
    bt.boute_route_grad(xs, mode, renorm, factor, idx.cuda(), g.cuda(), xs)  # in place
    assert torch.equal(xs, dx)


def tiny_choices(T, k):
    """The experts of tiny scores in turn, one row without a choice, one with a choice missing."""
    idx = torch.stack([(torch.arange(k) + r) % 6 + 2 for r in range(T)]).to(torch.int32)
    idx[2] = -1
    idx[3, 0] = -1
    return idx


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("E,k,pitch,shift", [(12, 1, 0, 0), (12, 6, 3, 1), (100, 4, 0, 0), (61, 5, 0, 1),
                                             (1000, 6, 8, 0)])
def test_gradient_of_logistic_scores_that_fp32_hardly_holds(renorm, E, k, pitch, shift):
    for dtype in ("f32", "bf16"):
        for factor in (1.0, 64.0):
            x = tiny_queries(E, dtype)
            tiny_gradient(x, SIG, tiny_choices(len(x), k), renorm, factor, E, pitch, shift)


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("E,k,pitch,shift", [(12, 1, 0, 0), (12, 6, 3, 1), (100, 4, 0, 0), (61, 5, 0, 1),
                                             (61, 2, 0, 3), (1000, 6, 8, 0), (333, 3, 1, 5)])
def test_gradient_of_softmax_scores_that_fp32_hardly_holds(renorm, dtype, E, k, pitch, shift):
    """A bias (or groups) has chosen experts far below the row's largest logit: weights that are 0
    have gradient 0."""
    for factor in (1.0, 64.0):
        x = tiny_queries(E, dtype)
        x[5, E - 1] = 3.0 if E > 12 else x[5, E - 1]   # the largest logit at the row's end
        x[6, -2:] = 1.5
        tiny_gradient(x, SOFT, tiny_choices(len(x), k), renorm, factor, E, pitch, shift)


def test_weights_and_gradient_agree_where_a_softmax_underflows():
    x = torch.tensor([[200.0, 0.0, 0.0, -1.0]]).cuda()
    bias = torch.tensor([-10.0, 0.0, 0.0, 0.0]).cuda()
    idx, w, _ = routed(x, bias, SOFT, 1, 1, 1, 2, True, 1.0, load=False)
    assert idx.tolist() == [[1, 2]] and w.tolist() == [[0.0, 0.0]]
    dx = torch.full_like(x, 9.0)
    bt.boute_route_grad(x, SOFT, True, 1.0, idx, torch.tensor([[1.0, -2.0]]).cuda(), dx)
    assert (dx == 0).all()


# ---------------------------------------------------------------- the bounds-checked build
CHILD = textwrap.dedent(r"""
    import sys
    sys.path.insert(0, ROOT); sys.path.insert(0, HERE)
    from paper_2602_10729_gb300 import boute as bt, build as bld
    bt.load(bld.build(debug=True))
    import test_gpu_answers as ta, test_gpu_answers_limits as tl, test_gpu_routing as tr

    ok = True
    def run(test, *a):
        global ok
        test(*a)
        r = bt.boute_bounds_report()
        if r is not None:
            ok = False
            print(test.__name__, a, f"VIOLATION unit={r[0]} line={r[1]} index={r[2]} extent={r[3]}")

    for T, V, scale, pitch, shift, ent in [(1, 1, 1.0, 0, 0, True), (4, 255, 1.25, 1, 5, True),
                                           (6, 1001, 1 / 0.7, 0, 3, True),
                                           (2, 50021, 1.0, 0, 0, True), (200, 300, 1.0, 0, 0, True)]:
        for dt in ("f32", "bf16"):
            run(ta.test_gradient_against_the_formula, dt, T, V, scale, pitch, shift, ent)
    run(tl.test_gradient_of_logits_far_from_zero, "bf16", 0.7, 4, 70001, True)
    run(ta.test_forward_many_short_rows, "f16", 7001, 8)
    run(tl.test_clusters_of_empty_answers)
    for E, k in ((48, 6), (256, 4), (256, 8), (200, 7)):
        for dt in ("f32", "bf16"):
            run(tr.test_many_queries_broken_rows, tr.SOFT, dt, E, k)
    for shape in tr.SHAPES + [(61, 190, 10, 4, 2, 6), (61, 192, 8, 4, 2, 6), (61, 254, 2, 1, 1, 5)]:
        run(tr.test_many_queries, tr.SIG, "f16", *shape)
    for T, E, k, pitch in [(1, 1, 1, 0), (4, 7, 3, 1), (37, 64, 2, 0), (5, 100, 10, 3), (3, 1024, 32, 0),
                           (9, 333, 6, 0), (1500, 48, 4, 8)]:
        for mode in (tr.SOFT, tr.SIG):
            for renorm in (True, False):
                run(tr.test_gradient_against_the_formula, mode, renorm, "bf16", T, E, k, pitch)
    for E, T, load in [(12, 9000, True), (250, 9000, True), (300, None, True)]:
        run(tl.test_choice_among_scores_that_fp32_hardly_holds, tr.SIG, False, E, T, load)
        run(tl.test_choice_among_scores_that_fp32_hardly_holds, tr.SOFT, True, E, T, load)
    print("BOUNDS_OK" if ok else "BOUNDS_BAD")
""")


def test_no_index_outside_its_extent():
    here = os.path.dirname(os.path.abspath(__file__))
    code = f"ROOT = {os.path.dirname(here)!r}; HERE = {here!r}\n" + CHILD
    p = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=900)
    assert p.returncode == 0, p.stdout + p.stderr
    assert "BOUNDS_OK" in p.stdout, p.stdout


# ---------------------------------------------------------------- very long answers
@pytest.mark.parametrize("lengths", [[100_000_000], [3] * 200_000 + [30_000_000] + [0, 2] * 500])
def test_means_of_very_long_answers(lengths):
    """Equal values, whose roundings all go the same way. Four positions join with 3 U, a thread's
    fours with 2 U (what an addition loses goes to the next), threads, warps and blocks in 21
    additions, then the count and the quotient: a mean is within 40 U of the value."""
    off = torch.tensor([0] + lengths).cumsum(0)
    T, Q = int(off[-1]), len(lengths)
    lp, ent = torch.full((T,), -0.1, device="cuda"), torch.full((T,), 0.3, device="cuda")
    s, n = torch.full((Q, 4), 9.0, device="cuda"), torch.zeros(Q, dtype=torch.int32, device="cuda")
    bt.boute_answer_scores(lp, ent, None, off.cuda(), s, n)
    assert n.tolist() == lengths
    some = s.cpu().double().numpy()[np.array(lengths) > 0]
    v = np.array([float(np.float32(-0.1)), float(np.float32(0.3))])
    assert (np.abs(some[:, [0, 2]] - v) <= 40 * U * np.abs(v)).all()
    assert (some[:, [1, 3]] == v).all()


# ---------------------------------------------------------------- long rows
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sums_of_long_rows_of_equal_terms(dtype):
    """Rows of one block, of one logit but for a few tokens of logit 0 that every warp meets: the
    roundings of equal terms all go the same way. A lane's 16 or 32 of a piece of the row join in two chains (8 U), up to
    64 pieces in another (32 U), chains, lanes and warps in 9 additions; the exponential's argument and
    the exponential have 6 U. ln s has an error of those 55 U and 2 U of its own size, 12: 80 U."""
    T, V = 700, 131072
    c = -(torch.arange(T) % 55 + 3).float() / 64
    x = torch.empty((T, V), dtype=DT[dtype], device="cuda")
    x[:] = c.cuda()[:, None]
    x[:, 5:4096:512] = 0.0
    t = torch.full((T,), 517, device="cuda")
    lp, H, lse, _, _ = forward(x, t, 1.0, 0)
    want = np.log(8.0 + (V - 8) * np.exp(c.double().numpy()))
    assert (np.abs(lse.cpu().double().numpy() - want) <= 80 * U).all()
    assert (np.abs(lp.cpu().double().numpy() + want) <= 80 * U).all()
