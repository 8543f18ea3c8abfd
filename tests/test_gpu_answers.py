"""Token log-probabilities, scores of answers, and their gradients, against
plain 64-bit forms: types, odd sizes, pitches and addresses, masks, rows
without a token left, NaN and infinities, ties, streams, long offsets.

Tolerances. z is rounded by definition; the difference z - m, the exponential's
argument and the logarithms carry a rounding each, of values up to D, the largest
m - z that an exponential sees (200 at most: beyond it is 0), and of a
log-probability's own size; a sum of n positive terms in any order errs like a
random walk of n roundings of U = 2^-24 (four deviations are allowed):
  tol = U (8 (2 + D) + 4 sqrt(V)),
for lse, which is rounded at its own size, 2 U |lse| more; for the entropy, whose
terms are weighted with up to 2 + ln V, times that. In the gradient p also has
the rounding of lse (rows with |lse| over 1024 do without it)."""
import numpy as np
import pytest
import torch

from _answers import U, answer_grad, answer_rows, token_grad_row, token_row
from paper_2602_10729_gb300 import boute as bt

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # one rounding to the type
F32, I64 = torch.float32, torch.int64


def placed(x, pitch=0, shift=0):
    """The same matrix on the device with `pitch` elements between rows, `shift` elements into a buffer."""
    T, V = x.shape
    buf = torch.full((T * (V + pitch) + shift,), 7.0, dtype=x.dtype, device="cuda")
    out = buf[shift:].view(T, V + pitch)[:, :V]
    out.copy_(x)
    return out


def logits(seed, T, V, dtype, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, V), generator=g) * spread
    t = torch.randint(0, V, (T,), generator=g)
    return x.to(DT[dtype]), t


def forward(x, t, scale, k, stream=None):
    T = x.shape[0]
    lp, H, lse = (torch.full((T,), 9.0, device="cuda") for _ in range(3))
    ti = torch.full((T, k), -7, dtype=I64, device="cuda") if k else None
    tv = torch.full((T, k), 9.0, device="cuda") if k else None
    bt.boute_token_logprobs(x, t, scale, lp, H, lse, ti, tv, stream)
    return lp, H, lse, ti, tv


def close(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf])
    fine = np.isfinite(want)
    assert np.isfinite(got[fine]).all()
    assert (np.abs(got - want)[fine] <= np.broadcast_to(tol, got.shape)[fine]).all(), \
        float(np.abs(got - want)[fine].max())


def tolerance(x, scale):
    z = x.astype(np.float64) * scale
    z = z[np.isfinite(z)]
    d = min(z.max() - z.min(), 200.0) if len(z) else 0.0
    return U * (8 * (2 + d) + 4 * np.sqrt(len(x)))


def check_forward(x, t, scale, k, out):
    lp, H, lse, ti, tv = (None if v is None else v.cpu().numpy() for v in out)
    xs = x.float().cpu().numpy()
    V = xs.shape[1]
    for r in range(xs.shape[0]):
        w = token_row(xs[r], scale, int(t[r]), k)
        tol = tolerance(xs[r], scale)
        close(lp[r], w[0], tol + 8 * U * (abs(w[0]) if np.isfinite(w[0]) else 0))
        close(H[r], w[1], tol * (2 + np.log(V)))
        close(lse[r], w[2], tol + 2 * U * (abs(w[2]) if np.isfinite(w[2]) else 0))
        if k:
            assert ti[r].tolist() == w[3], r
            tv_w = np.asarray(w[4])
            close(tv[r], tv_w, tol + 8 * U * np.where(np.isfinite(tv_w), np.abs(tv_w), 0))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V,k,scale,pitch,shift", [
    (1, 1, 1, 1.0, 0, 0), (3, 2, 2, 1.0, 0, 1), (5, 7, 7, 0.5, 2, 0), (2, 31, 5, 1.0, 0, 3),
    (4, 33, 32, 1.0, 0, 0), (3, 255, 20, 1.25, 1, 7), (3, 256, 8, 1.0, 0, 0),
    (3, 257, 32, 1.0, 0, 0), (7, 1000, 10, 1 / 0.7, 24, 0), (2, 4095, 1, 1.0, 1, 1),
    (2, 8192, 32, 1.0, 0, 0), (3, 8193, 3, 1.0, 0, 5), (1, 50021, 20, 1.0, 0, 0),
    (2, 50021, 5, 1.25, 3, 2), (1, 131072, 32, 1.0, 0, 0), (300, 513, 4, 1.0, 0, 0),
    (1, 300001, 32, 1.0, 0, 1), (2, 1 << 20, 7, 1.0, 0, 0), (40, 40001, 17, 1.0, 0, 0)])
def test_forward_sizes_types_and_places(dtype, T, V, k, scale, pitch, shift):
    x, t = logits(T * 31 + V, T, V, dtype)
    t[T // 2] = -1 if T > 1 else t[0]
    out = forward(placed(x, pitch, shift), t.cuda(), scale, k)
    check_forward(x, t, scale, k, out)


@pytest.mark.parametrize("dtype,V,k", [
    ("f32", 900, 0), ("bf16", 700, 4), ("f16", 7001, 8), ("bf16", 7001, 20), ("f32", 5003, 32),
    ("bf16", 2049, 1), ("f32", 513, 0)])
def test_forward_many_short_rows(dtype, V, k):
    T = 16001
    x, t = logits(V, 97, V, dtype)
    x[5, ::2] = -float("inf")
    x[7] = -float("inf")
    x[11, V // 3] = float("nan")
    x[13] = 0.5
    t[17] = -1
    rows = torch.arange(T) % 97
    out = forward(placed(x[rows], 1, 3), t[rows].cuda(), 1.25, k)
    some = torch.cat([torch.arange(97), T - 1 - torch.arange(97)])
    check_forward(x[rows[some]], t[rows[some]], 1.25, k,
                  tuple(None if v is None else v[some.cuda()] for v in out))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [5, 300, 9001, 131071])
def test_forward_masks_and_rows_without_a_token(dtype, V):
    T = 9
    x, t = logits(V, T, V, dtype)
    inf, low = float("inf"), torch.finfo(DT[dtype]).min
    x[0, ::2] = -inf                      # half masked
    x[1] = -inf                           # nothing left
    x[2] = low                            # the type's lowest value everywhere: uniform
    x[3] = -inf
    x[3, V // 2] = 1.5                    # one token left
    x[4, V - 1] = float("nan")
    x[5, 0] = inf
    x[6, : V - 1] = low                   # a mask by the lowest value, one token left
    x[7] = float(torch.finfo(DT[dtype]).max)
    t[0], t[3], t[6] = 0, V // 2, 0
    t[8] = V                              # out of the vocabulary
    k = min(V, 8)
    check_forward(x, t, 1.0, k, forward(placed(x, 1, 1), t.cuda(), 1.0, k))
    # nothing left and no token; NaN and no token; a masked token's log-probability
    t[1], t[4], t[0] = -1, -5, 0
    x[0, 0] = -inf
    check_forward(x, t, 1.0, k, forward(placed(x), t.cuda(), 1.0, k))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_scale_that_overflows(dtype):
    x, t = logits(5, 3, 700, dtype)
    x[0, 3] = -3e38                       # -inf once scaled: masked
    x[1, 5] = 3e38                        # +inf once scaled: no distribution
    x[2] = -3e38                          # every token masked
    check_forward(x, t, 2.0, 4, forward(x.cuda(), t.cuda(), 2.0, 4))


@pytest.mark.parametrize("V,k", [(64, 32), (1000, 32), (20011, 32), (70001, 20), (131072, 1)])
def test_alternatives_with_ties(V, k):
    """Values of few levels, constant rows, ascending and descending rows, -0 beside +0."""
    g = torch.Generator().manual_seed(V)
    x = torch.stack([torch.randint(0, 3, (V,), generator=g).float(), torch.zeros(V),
                     torch.arange(V).float() / V, -torch.arange(V).float() / V,
                     torch.where(torch.arange(V) % 2 == 0, -0.0, 0.0),
                     (torch.randn(V, generator=g) * 4).round() / 4])
    x[5, V // 3:] = -float("inf")
    t = torch.zeros(6, dtype=I64)
    for d in ("f32", "bf16"):
        y = x.to(DT[d])
        check_forward(y, t, 1.0, k, forward(y.cuda(), t.cuda(), 1.0, k))


def test_no_alternatives_and_no_rows():
    x, t = logits(3, 4, 333, "f32")
    check_forward(x, t, 1.0, 0, forward(x.cuda(), t.cuda(), 1.0, 0))
    before = bt.boute_launch_count()
    forward(torch.empty((0, 10), device="cuda"), torch.empty((0,), dtype=I64, device="cuda"), 1.0, 2)
    assert bt.boute_launch_count() == before


def test_rows_beyond_32_bit_offsets():
    """Five rows 2^30 elements apart: element offsets pass 2^31 and 2^32."""
    V, ld = 1003, 1 << 30
    buf = torch.empty((4 * ld + V,), dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((5, V), (ld, 1))
    y, t = logits(11, 5, V, "bf16")
    x.copy_(y)
    out = forward(x, t.cuda(), 1.0, 6)
    check_forward(y, t, 1.0, 6, out)
    g = torch.randn(5, generator=torch.Generator().manual_seed(1))
    bt.boute_token_logprobs_grad(x, t.cuda(), 1.0, out[2], out[1], g.cuda(), None, x)
    check_grad(y, t, 1.0, g, None, x, "bf16")


def test_another_stream_and_two_calls_at_once():
    x, t = logits(21, 64, 5003, "bf16")
    xs, ts = x.cuda(), t.cuda()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    a = forward(xs, ts, 1.0, 5)
    torch.cuda.synchronize()
    with torch.cuda.stream(s1):
        b = forward(xs, ts, 1.0, 5)
    with torch.cuda.stream(s2):
        c = forward(xs, ts, 1.0, 5)
    torch.cuda.synchronize()
    for u, v, w in zip(a, b, c):
        assert torch.equal(u, v) and torch.equal(u, w)


# ---------------------------------------------------------------- gradient
def check_grad(x, t, scale, g, gh, dx, dtype):
    got, xs = dx.float().cpu().numpy(), x.float().cpu().numpy()
    tiny = {"f32": 1e-38, "f16": 2.0 ** -25, "bf16": 1e-38}[dtype]  # of a subnormal result
    for r in range(xs.shape[0]):
        gr, hr = float(g[r]), 0.0 if gh is None else float(gh[r])
        want = token_grad_row(xs[r], scale, int(t[r]), gr, hr)
        z = xs[r].astype(np.float64) * scale
        V, fine = len(z), np.isfinite(z)
        m = z[fine].max() if fine.any() else 0.0
        d = np.where(fine, np.minimum(m - np.where(fine, z, m), 200.0), 200.0)
        # p's relative error (its exponent's absolute one), times the terms that it scales
        rel = tolerance(xs[r], scale) + 4 * U * min(abs(m), 1024.0)
        part = abs(gr) + abs(hr) * 2 * (2 + np.log(V) + d)
        tol = scale * rel * part * np.exp(-d)  # exp(-d) >= p
        tol = tol + np.abs(np.nan_to_num(want)) * (EPS[dtype] + 8 * U) + tiny
        close(got[r], want, tol)


def gradient(x, t, scale, g, gh, inplace=False, dx=None):
    lp, H, lse, _, _ = forward(x, t, scale, 0)
    dx = x if inplace else torch.full(x.shape, 5.0, dtype=x.dtype, device="cuda") if dx is None \
        else dx
    bt.boute_token_logprobs_grad(x, t, scale, lse, None if gh is None else H, g.cuda(),
                                 None if gh is None else gh.cuda(), dx)
    return dx


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V,scale,pitch,shift,ent", [
    (1, 1, 1.0, 0, 0, True), (3, 2, 1.0, 0, 1, True), (5, 37, 0.5, 3, 0, False),
    (4, 255, 1.25, 1, 5, True), (3, 1024, 1.0, 0, 0, True), (6, 1001, 1 / 0.7, 0, 3, True),
    (2, 8191, 1.0, 9, 1, False), (2, 50021, 1.0, 0, 0, True), (2, 131072, 1.25, 0, 0, True),
    (200, 300, 1.0, 0, 0, True)])
def test_gradient_against_the_formula(dtype, T, V, scale, pitch, shift, ent):
    x, t = logits(T * 7 + V, T, V, dtype)
    if T > 2:
        t[1] = -1
        x[2, ::3] = -float("inf")
    gen = torch.Generator().manual_seed(V)
    g, gh = torch.randn(T, generator=gen), torch.randn(T, generator=gen) if ent else None
    xs = placed(x, pitch, shift)
    out = placed(torch.zeros_like(x), (pitch * 2) % 5, (shift + 1) % 4)  # another pitch and place
    dx = gradient(xs, t.cuda(), scale, g, gh, dx=out)
    check_grad(x, t, scale, g, gh, dx, dtype)
    again = gradient(xs, t.cuda(), scale, g, gh, inplace=True)
    assert torch.equal(dx, again)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [6, 777, 20001])
def test_gradient_of_masked_and_broken_rows(dtype, V):
    x, t = logits(V, 7, V, dtype)
    inf = float("inf")
    x[0] = -inf
    x[1, 0] = float("nan")
    x[2, V - 1] = inf
    x[3] = -inf
    x[3, 2] = 0.25
    x[4] = torch.finfo(DT[dtype]).min
    t[0], t[3], t[5] = 1, 2, V
    g, gh = torch.ones(7), torch.full((7,), 0.5)
    check_grad(x, t, 1.0, g, gh, gradient(x.cuda(), t.cuda(), 1.0, g, gh), dtype)


def test_gradient_against_differences():
    """Central differences of the 64-bit log-probability and entropy, step 1e-5."""
    V, scale = 23, 1.3
    x, t = logits(8, 3, V, "f32", spread=1.5)
    t[1] = -1
    g, gh = torch.tensor([1.0, 2.0, -0.7]), torch.tensor([0.3, -1.0, 0.0])
    dx = gradient(x.cuda(), t.cuda(), scale, g, gh).cpu().numpy()

    def loss(row, r):
        z = row * float(np.float32(scale))
        lse = np.log(np.exp(z).sum())
        lp = z - lse
        H = -(np.exp(lp) * lp).sum()
        return (float(g[r]) * lp[t[r]] if t[r] >= 0 else 0.0) + float(gh[r]) * H

    for r in range(3):
        for j in range(V):
            row = x[r].double().numpy()
            d = np.zeros(V)
            d[j] = 1e-5
            want = (loss(row + d, r) - loss(row - d, r)) / 2e-5
            assert abs(dx[r, j] - want) < 1e-5


# ---------------------------------------------------------------- scores of answers
def answers(seed, lengths, before=0, after=0, skip=0.1):
    g = torch.Generator().manual_seed(seed)
    off = np.concatenate([[0], np.cumsum(lengths)]) + before
    T = int(off[-1]) + after
    lp = -torch.rand(T, generator=g) * 8
    ent = torch.rand(T, generator=g) * 5
    t = torch.where(torch.rand(T, generator=g) < skip, -1, 3)
    return lp, ent, t, torch.as_tensor(off)


def scored(lp, ent, t, off):
    Q = len(off) - 1
    s = torch.full((Q, 4), 9.0, device="cuda")
    n = torch.full((Q,), -3, dtype=torch.int32, device="cuda")
    bt.boute_answer_scores(lp.cuda(), ent.cuda(), None if t is None else t.cuda(), off.cuda(), s, n)
    return s.cpu().numpy(), n.cpu().numpy()


LENGTHS = {"one": [1], "tiny": [1, 0, 2, 3, 0, 0, 31, 32, 33], "mixed": [5, 700, 0, 255, 256, 257, 3],
           "long": [40001], "wide": list(np.arange(600) % 23), "few-long": [9000, 1, 20011, 0],
           "one-among-many": [3] * 500 + [30000] + [2] * 500, "none": [0, 0, 0]}


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("masked", [True, False])
def test_scores_of_answers(name, masked):
    lp, ent, t, off = answers(len(name), LENGTHS[name], before=3, after=5)
    if masked and len(LENGTHS[name]) > 3:
        t[int(off[2]):int(off[4])] = -1   # an answer whose positions hold no token
    t = t if masked else None
    got, n = scored(lp, ent, t, off)
    want, cnt = answer_rows(lp.numpy(), ent.numpy(), None if t is None else t.numpy(), off.numpy())
    assert n.tolist() == cnt.tolist()
    assert np.array_equal(got[:, [1, 3]], want[:, [1, 3]].astype(np.float32))
    # a sum of n roundings of values up to 8 over n, and the quotient's own rounding
    tol = U * 8 * (4 + 4 * np.sqrt(np.maximum(cnt, 1)))[:, None]
    close(got[:, [0, 2]], want[:, [0, 2]], tol)


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("masked", [True, False])
def test_gradient_of_the_scores(name, masked):
    lp, ent, t, off = answers(len(name) + 50, LENGTHS[name], before=2, after=4)
    lp, ent = (lp * 4).round() / 4, (ent * 4).round() / 4  # ties: the first position
    t = t if masked else None
    g = torch.randn((len(off) - 1, 4), generator=torch.Generator().manual_seed(5))
    gl, gh = torch.full_like(lp, 9.0).cuda(), torch.full_like(lp, 9.0).cuda()
    bt.boute_answer_scores_grad(lp.cuda(), ent.cuda(), None if t is None else t.cuda(), off.cuda(),
                                g.cuda(), gl, gh)
    wl, wh = answer_grad(lp.numpy(), ent.numpy(), None if t is None else t.numpy(), off.numpy(),
                         g.double().numpy())
    close(gl.cpu().numpy(), wl, 4 * U * 10)  # |g| < 5: a quotient and a sum of two
    close(gh.cpu().numpy(), wh, 4 * U * 10)


def test_scores_of_nan_and_infinite_positions():
    lp = torch.tensor([-1.0, float("nan"), -3.0, -float("inf"), -1.0, 0.0])
    ent = torch.tensor([0.5, 1.0, float("nan"), 2.0, 3.0, float("inf")])
    off = torch.tensor([0, 3, 6])
    s, n = scored(lp, ent, None, off)
    assert n.tolist() == [3, 3]
    assert np.isnan(s[0]).all()
    assert s[1].tolist() == [-np.inf, -np.inf, np.inf, np.inf]
    gl, gh = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    g = torch.tensor([[0.0, 1.0, 0.0, 2.0], [3.0, 1.0, 0.0, 2.0]])
    bt.boute_answer_scores_grad(lp.cuda(), ent.cuda(), None, off.cuda(), g.cuda(), gl, gh)
    assert gl.cpu().tolist() == [0, 1, 0, 2, 1, 1]
    assert gh.cpu().tolist() == [0, 0, 2, 0, 0, 2]


def test_scores_without_positions_and_without_answers():
    empty = torch.empty((0,))
    s, n = scored(empty, empty, None, torch.zeros(4, dtype=I64))
    assert (s == 0).all() and n.tolist() == [0, 0, 0]
    gl, gh = torch.full((5,), 9.0, device="cuda"), torch.full((5,), 9.0, device="cuda")
    v = torch.ones(5, device="cuda")
    bt.boute_answer_scores_grad(v, v, None, torch.zeros(1, dtype=I64, device="cuda"),
                                torch.empty((0, 4), device="cuda"), gl, gh)
    assert (gl == 0).all() and (gh == 0).all()


def test_offsets_out_of_range_are_cut():
    lp, ent, t, _ = answers(4, [10])
    s, n = scored(lp, ent, None, torch.tensor([-5, 4, 3, 999]))
    assert n.tolist() == [4, 0, 7]
