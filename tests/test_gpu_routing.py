"""Routing of queries to experts and its gradient against plain 64-bit forms.

The choice is compared where it hangs on more than rounding: a score carries a
few roundings (U = 2^-24 each), so queries whose 64-bit scores differ by more
than 0 but less than 64 U of the largest are left out (equal scores are not:
they go to the lowest index). Weights and gradients: a score's relative error is
at most U (16 + 2 min(max |x|, 200) + 4 sqrt(E)) (exponential, its argument, the
softmax's sum), a renormalised weight's twice that."""
import numpy as np
import pytest
import torch

from _answers import U, route_grad_row, route_row, scores
from paper_2602_10729_gb300 import boute as bt
from test_gpu_answers import DT, EPS, close, placed

pytestmark = pytest.mark.gpu

SOFT, SIG = bt.BOUTE_ROUTE_SOFTMAX, bt.BOUTE_ROUTE_SIGMOID


def queries(seed, T, E, dtype, spread=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, E), generator=g) * spread).to(DT[dtype])


def routed(x, bias, mode, G, keep, gtop, k, renorm, factor, load=True, stream=None):
    T, E = x.shape
    idx = torch.full((T, k), -9, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), 9.0, device="cuda")
    ld = torch.full((E,), 99, dtype=torch.int32, device="cuda") if load else None
    bt.boute_route(x, bias, mode, G, keep, gtop, renorm, factor, idx, w, ld, stream)
    return idx, w, ld


def rel_tol(x):
    v = np.abs(x[np.isfinite(x)]).astype(np.float64)
    return U * (16 + 2 * min(v.max(initial=0), 200.0) + 4 * np.sqrt(len(x)))


def check(x, bias, mode, G, keep, gtop, k, renorm, factor, out):
    idx, w, ld = (None if v is None else v.cpu().numpy() for v in out)
    xs = x.float().cpu().numpy()
    b = None if bias is None else bias.cpu().numpy()
    left_out = 0
    for r in range(len(xs)):
        wi, ww, gap = route_row(xs[r], b, mode, G, keep, gtop, k, renorm, factor)
        s = scores(xs[r], mode)
        if s is not None:
            big = s.max() + (0 if b is None else np.abs(b[np.isfinite(b)]).max(initial=0))
            if gap < 64 * U * big:
                left_out += 1
                continue
        assert idx[r].tolist() == wi, (r, idx[r].tolist(), wi)
        close(w[r], ww, 2 * rel_tol(xs[r]) * np.abs(np.nan_to_num(ww)) + 1e-37)
    assert left_out <= max(2, len(xs) // 50)
    if ld is not None:
        got = idx[idx >= 0]
        assert ld.tolist() == np.bincount(got, minlength=xs.shape[1]).tolist()


SHAPES = [  # T, E, G, keep, group_top, k
    (1, 1, 1, 1, 1, 1), (3, 2, 1, 1, 1, 2), (5, 7, 1, 1, 1, 3), (33, 64, 1, 1, 1, 2),
    (50, 60, 6, 2, 1, 4), (70, 192, 8, 4, 2, 6), (9, 96, 32, 5, 2, 7), (17, 33, 1, 1, 1, 32),
    (4, 320, 5, 5, 1, 10), (21, 257, 1, 1, 1, 8), (6, 1024, 16, 3, 2, 32), (5, 1000, 8, 1, 1, 9),
    (200, 128, 4, 4, 2, 4), (12, 32, 32, 7, 2, 7), (3001, 40, 4, 2, 2, 5)]


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,E,G,keep,gtop,k", SHAPES)
def test_route_sizes_and_types(mode, dtype, T, E, G, keep, gtop, k):
    x = queries(T * 3 + E, T, E, dtype)
    g = torch.Generator().manual_seed(E)
    bias = torch.randint(-100, 100, (E,), generator=g).float() * 1e-3 if mode == SIG or T % 2 else None
    pitch, shift = T % 5, E % 3
    a = (None if bias is None else bias.cuda(), mode, G, keep, gtop, k, E % 2 == 0, 2.5)
    out = routed(placed(x, pitch, shift), *a)
    check(x, *a, out)


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("G,keep", [(1, 1), (4, 2)])
def test_experts_out_of_service_and_broken_rows(mode, G, keep):
    T, E, k = 12, 48, 6
    x = queries(5, T, E, "f32")
    inf = float("inf")
    x[0] = -inf                      # nobody in service
    x[1, 2:] = -inf                  # fewer than k
    x[2, 12:36] = -inf               # groups without anyone
    x[3, 7] = float("nan")
    x[4, 9] = inf
    x[5] = 0.25                      # all equal: the lowest indices
    x[6] = torch.finfo(torch.float32).min
    x[7, 1:] = -200.0                # logistic scores that underflow
    x[8] = -200.0
    x[9, ::2] = -inf
    for bias in (None, torch.zeros(E), torch.where(torch.arange(E) % 3 == 0, -inf, 0.125)):
        b = None if bias is None else bias.cuda()
        for renorm in (True, False):
            a = (b, mode, G, keep, 2, k, renorm, 1.0)
            check(x, *a, routed(x.cuda(), *a))
    nan_bias = torch.zeros(E)
    nan_bias[::5] = float("nan")
    a = (nan_bias.cuda(), mode, G, keep, 1, k, True, 1.0)
    check(x, *a, routed(x.cuda(), *a))


def test_ties_go_to_the_lowest_index():
    g = torch.Generator().manual_seed(9)
    x = torch.randint(0, 3, (400, 72), generator=g).float()
    for dtype in ("f32", "bf16"):
        for G, keep, gtop in ((1, 1, 1), (8, 3, 2), (12, 5, 1)):
            for mode in (SOFT, SIG):
                a = (None, mode, G, keep, gtop, 9, True, 1.0)
                check(x.to(DT[dtype]), *a, routed(x.to(DT[dtype]).cuda(), *a))


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("T,E,G,keep,gtop,k", [  # lists as long as a lane's values, and groups that
    (300, 64, 1, 1, 1, 8), (300, 50, 1, 1, 1, 32), (300, 128, 1, 1, 1, 12),  # 1 to 16 lanes hold
    (300, 100, 1, 1, 1, 20), (300, 60, 6, 3, 1, 8), (300, 64, 8, 3, 2, 4), (300, 128, 8, 4, 2, 6),
    (300, 240, 5, 2, 2, 9), (300, 256, 2, 1, 1, 30), (300, 160, 20, 3, 2, 20),
    (40, 480, 3, 2, 2, 32), (40, 1024, 32, 2, 1, 32), (300, 168, 8, 5, 2, 9)])
def test_long_choices_and_groups_of_lanes(mode, T, E, G, keep, gtop, k):
    g = torch.Generator().manual_seed(E + k)
    bias = torch.randint(-100, 100, (E,), generator=g).float() * 1e-3
    x = queries(E, T, E, "bf16")
    x[::7, ::3] = float("-inf")
    ties = torch.randint(0, 3, (T, E), generator=g).float()
    for v, b in ((x, None), (x, bias), (ties, None)):
        a = (None if b is None else b.cuda(), mode, G, keep, gtop, k, True, 1.0)
        check(v, *a, routed(v.cuda(), *a))


def check_many(x, *a, T=4999, pitch=0, shift=0):
    """The queries over and over, enough to fill the device: equal ones are treated alike."""
    rows = torch.arange(T) % len(x)
    i, w, ld = routed(placed(x[rows], pitch, shift), *a)
    rows = rows.cuda()
    assert torch.equal(i, i[:len(x)][rows])
    assert torch.equal(w.view(torch.int32), w[:len(x)][rows].view(torch.int32))
    assert ld.tolist() == torch.bincount(i[i >= 0].long(), minlength=x.shape[1]).tolist()
    check(x, *a, (i[:len(x)], w[:len(x)], None))


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,E,G,keep,gtop,k", SHAPES + [
    (61, 256, 1, 1, 1, 4), (61, 256, 8, 4, 2, 8), (61, 192, 8, 4, 2, 6), (61, 190, 10, 4, 2, 6),
    (61, 160, 5, 2, 2, 6), (61, 160, 10, 3, 1, 3), (61, 128, 8, 2, 2, 8), (61, 64, 8, 3, 1, 8),
    (61, 61, 1, 1, 1, 8), (61, 254, 2, 1, 1, 5), (61, 8, 1, 1, 1, 8), (61, 129, 3, 1, 2, 1)])
def test_many_queries(mode, dtype, T, E, G, keep, gtop, k):
    x = queries(T * 5 + E, min(T, 19), E, dtype, 0.7)
    x[::9, ::2] = float("-inf")
    g = torch.Generator().manual_seed(E)
    bias = (torch.randint(-100, 100, (E,), generator=g).float() * 1e-3).cuda()
    for b, renorm in ((None, True), (bias, E % 2 == 0), (None, False)):
        check_many(x, b, mode, G, keep, gtop, k, renorm, 2.5, pitch=E % 3, shift=k % 2)
    ties = torch.randint(0, 3, x.shape, generator=g).to(DT[dtype])
    check_many(ties, None, mode, G, keep, gtop, k, True, 1.0)


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("E,k", [(48, 6), (100, 3), (256, 4), (256, 8), (200, 7)])
def test_many_queries_broken_rows(mode, dtype, E, k):
    x = queries(E, 18, E, dtype)
    inf, low = float("inf"), torch.finfo(DT[dtype]).min
    x[0] = -inf                      # nobody in service
    x[1, 2:] = -inf                  # fewer than k
    x[2, 12:36] = -inf
    x[3, 7] = float("nan")
    x[4, 9] = inf
    x[5] = 0.25                      # all equal: the lowest indices
    x[6] = low
    x[7, 1:] = low
    x[8] = -200.0
    x[9, ::2] = -inf
    x[10] = float("nan")
    x[11] = 0.0
    x[11, ::2] = -0.0                # one value
    x[12] = torch.arange(E).to(DT[dtype]) / 64
    x[13] = -torch.arange(E).to(DT[dtype]) / 64
    x[14] = 1.0                      # all of the largest in one lane
    x[14, 16:24] = 2.0
    x[15, :40] = -inf
    x[16, 40:] = -inf
    off = torch.where(torch.arange(E) % 3 == 0, -inf, 0.125)
    for b in (None, torch.zeros(E), off):
        for G, keep, renorm in ((1, 1, True), (1, 1, False), (4, 2, True)):
            if k <= keep * (E // G):
                check_many(x, None if b is None else b.cuda(), mode, G, keep, 2, k, renorm, 1.0)


def test_load_is_written_and_optional():
    x = queries(2, 100, 16, "bf16").cuda()
    a = (None, SOFT, 1, 1, 1, 3, True, 1.0)
    i1, w1, l1 = routed(x, *a)
    i2, w2, l2 = routed(x, *a, load=False)
    assert l2 is None and torch.equal(i1, i2) and torch.equal(w1, w2)
    assert int(l1.sum()) == 300
    _, _, l0 = routed(x[:0], *a)
    assert l0.tolist() == [0] * 16


def test_another_stream():
    x = queries(4, 777, 100, "f16").cuda()
    a = (None, SIG, 4, 2, 2, 5, True, 1.0)
    want = routed(x, *a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = routed(x, *a)
    s.synchronize()
    for u, v in zip(want, got):
        assert torch.equal(u, v)


# ---------------------------------------------------------------- gradient
def grad_tol(x, mode, idx, g, renorm, factor, dtype):
    """Of one row: the relative error of the scores times the terms that they scale, and the
    output's rounding."""
    s = scores(x, mode)
    on = [r for r, e in enumerate(idx) if e >= 0]
    if s is None or not on:
        return np.zeros(len(x)) + 1e-38
    e = np.array([idx[r] for r in on])
    gm = np.abs(np.array([g[r] for r in on])).max() * factor
    if renorm:
        S = s[e].sum()
        gm = 2 * gm / S if S > 0 else 0.0
    want = np.abs(route_grad_row(x, mode, idx, g, renorm, factor))
    hit = np.isin(np.arange(len(x)), e) if mode == SIG else np.ones(len(x), bool)
    terms = gm * s * (hit if mode == SIG else (hit + s[e].sum()))
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-37
    return 4 * rel_tol(x) * terms + want * EPS[dtype] * 1.01 + tiny


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,E,k,pitch", [(1, 1, 1, 0), (4, 7, 3, 1), (37, 64, 2, 0), (5, 100, 10, 3),
                                         (3, 1024, 32, 0), (9, 333, 6, 0), (1500, 48, 4, 8)])
def test_gradient_against_the_formula(mode, renorm, dtype, T, E, k, pitch):
    x = queries(T + E, T, E, dtype)
    if T > 3:
        x[2, : E // 2] = -float("inf")
    xs = placed(x, pitch, 1)
    idx, _, _ = routed(xs, None, mode, 1, 1, 1, k, renorm, 2.0, load=False)
    if T > 3:
        idx[1] = -1                       # a query without a choice
        idx[3, 0] = -1                    # a choice that does not exist
    g = torch.randn((T, k), generator=torch.Generator().manual_seed(T))
    dx = placed(torch.zeros_like(x), (pitch * 3) % 4, 2)
    bt.boute_route_grad(xs, mode, renorm, 2.0, idx, g.cuda(), dx)
    got, xf, ii = dx.float().cpu().numpy(), x.float().numpy(), idx.cpu().numpy()
    for r in range(T):
        a = (mode, ii[r].tolist(), g[r].tolist(), renorm, 2.0)
        close(got[r], route_grad_row(xf[r], *a), grad_tol(xf[r], *a, dtype))
    bt.boute_route_grad(xs, mode, renorm, 2.0, idx, g.cuda(), xs)  # in place
    assert torch.equal(xs, dx)


@pytest.mark.parametrize("mode", [SOFT, SIG])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(mode, renorm):
    """Central differences of the 64-bit weights with the choice held, step 1e-5."""
    E, k = 11, 4
    x = queries(3, 2, E, "f32")
    idx, _, _ = routed(x.cuda(), None, mode, 1, 1, 1, k, renorm, 1.5, load=False)
    g = torch.randn((2, k), generator=torch.Generator().manual_seed(7))
    dx = torch.empty_like(x).cuda()
    bt.boute_route_grad(x.cuda(), mode, renorm, 1.5, idx, g.cuda(), dx)

    def loss(row, r):
        s = scores(row, mode)[idx[r].cpu().numpy()]
        return float((g[r].double().numpy() * 1.5 * (s / s.sum() if renorm else s)).sum())

    for r in range(2):
        for j in range(E):
            d = np.zeros(E)
            d[j] = 1e-5
            row = x[r].double().numpy()
            want = (loss(row + d, r) - loss(row - d, r)) / 2e-5
            assert abs(float(dx[r, j]) - want) < 1e-5


def test_gradient_of_scores_that_underflow_and_of_broken_rows():
    x = torch.full((3, 8), -200.0)
    x[1, 3] = float("nan")
    x[2] = -float("inf")
    idx, w, _ = routed(x.cuda(), None, SIG, 1, 1, 1, 3, True, 1.0, load=False)
    assert idx.cpu().tolist() == [[0, 1, 2], [-1] * 3, [-1] * 3]
    assert w[0].tolist() == [0, 0, 0] and w[2].tolist() == [0, 0, 0] and bool(w[1].isnan().all())
    dx = torch.full_like(x, 9.0).cuda()
    bt.boute_route_grad(x.cuda(), SIG, True, 1.0, idx, torch.ones(3, 3).cuda(), dx)
    assert (dx == 0).all()
