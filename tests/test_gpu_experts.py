"""The choices of a routing sorted by expert, the queries' rows there and back, and the gradients,
against plain forms in 64 bits: types, odd sizes, pitches and addresses, queries without a
choice, places beyond the rows, every sort's sizes, streams and graphs.

Tolerances. A sum of n terms a_i taken with one rounding (U = 2^-24, relative to a partial sum) a
step is off by n U sum |a_i| at most; a product that is rounded before it is added, or written,
adds one of its own. A lane sums one element in TEAM (8 or 32) of a dot product, and log2(TEAM)
more additions join the lanes. Rounding to the type is half a step, EPS, relative, or half of the
type's smallest number where the value is below its normal range."""
import numpy as np
import pytest
import torch

from paper_2602_10729_gb300 import boute as bt

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
I32, F32 = torch.int32, torch.float32


def placed(x, pitch=0, shift=0, fill=float("nan")):
    """The same matrix on the device with `pitch` elements between rows, `shift` elements into a buffer."""
    R, D = x.shape
    buf = torch.full((R * (D + pitch) + shift,), fill, dtype=x.dtype, device="cuda")
    out = buf[shift:].view(R, D + pitch)[:, :D]
    out.copy_(x)
    return out


def n64(t):
    return t.detach().cpu().double().numpy()


def choices(seed, T, k, E, none=0.1, twice=False):
    """T x k choices, k different experts each (any, with `twice`), some queries and choices without."""
    r = np.random.default_rng(seed)
    if twice:
        idx = r.integers(0, E, (T, k))
    else:
        idx = np.argsort(r.random((T, E)), axis=1)[:, :k]
    idx = np.where(r.random((T, k)) < none / 2, -1, idx)
    idx[r.random(T) < none / 2] = -1
    return idx.astype(np.int32)


def plain_sort(idx, E):
    flat = idx.reshape(-1)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(key, kind="stable")
    n = int((key < E).sum())
    source = np.where(np.arange(len(flat)) < n, order, -1)
    place = np.full(len(flat), -1)
    place[order[:n]] = np.arange(n)
    return np.searchsorted(key[order], np.arange(E + 1)), source, place.reshape(idx.shape)


def sort(idx, E, stream=None):
    T, k = idx.shape
    offsets, source = (torch.full((n,), -9, dtype=I32, device="cuda") for n in (E + 1, T * k))
    place = torch.full((T, k), -9, dtype=I32, device="cuda")
    bt.boute_expert_sort(idx, offsets, source, place, stream)
    return offsets, source, place


def check_sort(idx, E):
    got = sort(torch.from_numpy(idx).cuda(), E)
    for g, w in zip(got, plain_sort(idx, E)):
        assert np.array_equal(g.cpu().numpy(), w)
    return got


@pytest.mark.parametrize("T,k,E", [
    (0, 2, 5), (1, 1, 1), (1, 8, 8), (32, 2, 64), (33, 3, 3), (511, 8, 1024), (512, 8, 61),
    (513, 8, 61), (4099, 6, 61), (4096, 8, 1024), (4097, 8, 1024), (10923, 3, 256), (32769, 1, 7),
    (5000, 32, 1024), (100003, 5, 257), (300000, 4, 2), (262144, 4, 256)])
def test_sort(T, k, E):
    check_sort(choices(T + E, T, k, E, twice=T > 50000), E)


@pytest.mark.parametrize("T", [40, 3000, 60000])
def test_sort_of_one_expert_of_none_and_of_numbers_that_are_none(T):
    for idx in (np.zeros((T, 2)), np.full((T, 2), 6), np.full((T, 2), -1)):
        check_sort(idx.astype(np.int32), 7)
    r = np.random.default_rng(T)
    odd = np.array([-1, 0, 6, 7, 8, 1 << 20, 2 ** 31 - 1, -2 ** 31], np.int32)
    check_sort(odd[r.integers(0, len(odd), (T, 3))], 7)


@pytest.mark.parametrize("T", [100, 9000])
def test_sort_of_an_expert_named_twice_keeps_the_choices_order(T):
    idx = np.random.default_rng(5).integers(0, 3, (T, 4)).astype(np.int32)
    _, source, place = check_sort(idx, 3)
    assert (place.cpu().numpy()[idx[:, 0] == idx[:, 1]][:, :2] @ [1, -1] < 0).all()


# ---- rows
ROWS = [  # T, k, E, D, dtype, pitch, shift
    (1, 1, 2, 1, "f16", 0, 0), (1, 2, 3, 4096, "bf16", 0, 0), (7, 3, 5, 24, "f32", 0, 0),
    (65, 2, 9, 7, "bf16", 1, 1), (33, 5, 6, 1001, "f16", 3, 0), (33, 5, 6, 1001, "bf16", 2, 5),
    (40, 8, 16, 1024, "bf16", 8, 0), (19, 4, 4, 515, "f32", 0, 1), (9, 2, 32, 8192, "f32", 4, 0),
    (300, 1, 4, 64, "f16", 4, 4), (50, 32, 40, 130, "bf16", 0, 0), (21, 9, 12, 2050, "f16", 0, 2),
    (5, 3, 7, 8191, "bf16", 0, 0), (1025, 7, 11, 8, "f16", 0, 0), (100, 2, 4, 16, "f32", 0, 0)]


def setup(T, k, E, D, dtype, pitch, shift, seed=0):
    r = np.random.default_rng(seed + T * 7 + D)
    g = torch.Generator().manual_seed(seed + T + D)
    idx = choices(seed + T, T, k, E)
    _, _, place = plain_sort(idx, E)
    w = r.random((T, k)).astype(np.float32) + 0.1
    w[place < 0] = np.nan  # (boute_route gives NaN to a query that has no choice)
    randn = lambda n: torch.randn((n, D), generator=g).to(DT[dtype])
    dev = lambda x: placed(x, pitch, shift)
    return place, w, randn, dev


def rounded(want, slack, dtype):
    """What a value computed within `slack` of `want` may be off by after one rounding to the type."""
    return slack + EPS[dtype] * (np.abs(want) + slack) + TINY[dtype]


@pytest.mark.parametrize("T,k,E,D,dtype,pitch,shift", ROWS)
def test_dispatch_and_its_gradient(T, k, E, D, dtype, pitch, shift):
    place, _, randn, dev = setup(T, k, E, D, dtype, pitch, shift)
    N, x, g = T * k, randn(T), randn(T * k)
    was = randn(N)
    rows = dev(was)
    P = torch.from_numpy(place.astype(np.int32)).cuda()
    bt.boute_expert_dispatch(dev(x), P, rows)
    want = was.clone()
    for c, p in enumerate(place.reshape(-1)):
        if p >= 0:
            want[p] = x[c // k]
    assert torch.equal(rows.cpu(), want)  # (those of no choice as they were)
    used = np.zeros(N, bool)
    used[place[place >= 0]] = True
    g[~torch.from_numpy(used)] = float("nan")  # (nor are theirs read)
    dx = dev(randn(T))
    bt.boute_expert_dispatch_grad(dev(g), P, dx)
    v = np.where((place >= 0)[:, :, None], n64(g)[np.maximum(place, 0)], 0.0)
    want = v.sum(1)
    tol = rounded(want, k * U * np.abs(v).sum(1), dtype)
    assert (np.abs(n64(dx) - want) <= tol).all()


@pytest.mark.parametrize("T,k,E,D,dtype,pitch,shift", ROWS)
def test_combine_and_its_gradient(T, k, E, D, dtype, pitch, shift):
    place, w, randn, dev = setup(T, k, E, D, dtype, pitch, shift, 1)
    N, rows, go = T * k, randn(T * k), randn(T)
    on = place >= 0
    used = np.zeros(N, bool)
    used[place[on]] = True
    rows[~torch.from_numpy(used)] = float("nan")
    P, W = torch.from_numpy(place.astype(np.int32)).cuda(), torch.from_numpy(w).cuda()
    out, x = dev(randn(T)), dev(rows)
    bt.boute_expert_combine(x, P, W, out)
    v = np.where(on[:, :, None], n64(rows)[np.maximum(place, 0)], 0.0)
    w64 = np.where(on, w, 0.0).astype(np.float64)
    a = w64[:, :, None] * v
    want = a.sum(1)
    assert (np.abs(n64(out) - want) <= rounded(want, k * U * np.abs(a).sum(1), dtype)).all()

    g_rows, g_weight = dev(randn(N)), torch.full((T, k), 9.0, device="cuda")
    before = g_rows.clone()
    bt.boute_expert_combine_grad(dev(go), x, P, W, g_rows, g_weight)
    a = n64(go)[:, None] * v
    want = a.sum(2)
    tol = (D / 8 + 16) * U * np.abs(a).sum(2)
    assert (np.abs(n64(g_weight) - want) <= tol).all()
    assert (n64(g_weight)[~on] == 0).all()
    got = n64(g_rows)
    want = (w64[:, :, None] * n64(go)[:, None])[on]
    assert (np.abs(got[place[on]] - want) <= rounded(want, U * np.abs(want), dtype)).all()
    assert torch.equal(g_rows[~torch.from_numpy(used).cuda()], before[~torch.from_numpy(used).cuda()])
    # in place
    again = torch.full((T, k), 9.0, device="cuda")
    x[~torch.from_numpy(used).cuda()] = before[~torch.from_numpy(used).cuda()]
    bt.boute_expert_combine_grad(dev(go), x, P, W, x, again)
    assert torch.equal(again, g_weight) and torch.equal(x, g_rows)


@pytest.mark.parametrize("R", [0, 1, 10, 1000])
def test_places_beyond_the_rows_are_none(R):
    place = torch.tensor([[0, 12], [9, -5], [10, 2 ** 31 - 1], [-2 ** 31, 999]], dtype=I32).cuda()
    T, k, D = 4, 2, 40
    x, w = torch.randn((T, D), device="cuda"), torch.rand((T, k), device="cuda")
    buf = torch.full((R + 2, D), 5.0, device="cuda")
    rows = buf[:R]
    bt.boute_expert_dispatch(x, place, rows)
    want, on = torch.full((R + 2, D), 5.0), (place >= 0) & (place < R)
    for t in range(T):
        for i in range(k):
            if on[t, i]:
                want[place[t, i]] = x[t].cpu()
    assert torch.equal(buf.cpu(), want)
    out, dx = torch.full((T, D), 7.0, device="cuda"), torch.full((T, D), 7.0, device="cuda")
    bt.boute_expert_combine(rows, place, w, out)
    bt.boute_expert_dispatch_grad(rows, place, dx)
    s, n = (w * on).sum(1, keepdim=True), on.sum(1, keepdim=True)
    assert torch.allclose(out, s * x, rtol=1e-6, atol=1e-6) and torch.allclose(dx, n * x, rtol=1e-6)
    g_rows, g_weight = torch.full((R + 2, D), 5.0, device="cuda"), torch.full((T, k), 7.0, device="cuda")
    bt.boute_expert_combine_grad(x, rows, place, w, g_rows[:R], g_weight)
    assert torch.equal(g_weight == 0, ~on) and (g_rows[R:] == 5.0).all()


def test_infinities_and_nan_stay_with_their_queries():
    T, k, D = 6, 2, 100
    idx = torch.arange(T * k, dtype=I32, device="cuda").view(T, k) % 3
    _, _, place = sort(idx, 3)
    rows = torch.ones((T * k, D), dtype=torch.bfloat16, device="cuda")
    rows[place[1, 0], 3], rows[place[2, 1], 4] = float("inf"), float("nan")
    out = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    w = torch.ones((T, k), device="cuda")
    bt.boute_expert_combine(rows, place, w, out)
    assert out[1, 3] == float("inf") and out[2, 4].isnan() and int((out != 2).sum()) == 2


def test_gradients_against_differences():
    """Of f = <u, combine(rows)> + <v, dispatch(x)>, which is linear in each: the difference is
    the gradient up to roundings (of T k D terms of order 1, in fp32)."""
    T, k, E, D = 13, 3, 5, 37
    idx = torch.from_numpy(choices(2, T, k, E)).cuda()
    _, _, place = sort(idx, E)
    N, new = T * k, lambda *s: torch.randn(s, device="cuda")
    x, rows, w, u, v = new(T, D), new(N, D), new(T, k).abs(), new(T, D), new(N, D)
    w[place < 0] = 0.0
    used = torch.zeros(N, dtype=torch.bool, device="cuda")
    used[place[place >= 0].long()] = True

    def f(x, rows, w):
        out, sent = torch.zeros((T, D), device="cuda"), torch.zeros((N, D), device="cuda")
        bt.boute_expert_combine(rows, place, w, out)
        bt.boute_expert_dispatch(x, place, sent)
        return ((u.double() * out).sum() + (v.double() * sent).sum()).item()

    g_rows, g_w, dx = torch.zeros((N, D), device="cuda"), new(T, k), new(T, D)
    bt.boute_expert_combine_grad(u, rows, place, w, g_rows, g_w)
    bt.boute_expert_dispatch_grad(v, place, dx)
    d = [new(T, D), new(N, D), new(T, k) * (place >= 0)]
    for j, (a, g) in enumerate(zip((x, rows, w), (dx, g_rows, g_w))):
        at = [x, rows, w]
        at[j] = a + d[j]
        up = f(*at)
        at[j] = a - d[j]
        slope = (up - f(*at)) / 2
        want = (g.double() * d[j]).sum().item()
        scale = float(T * k * D) ** 0.5
        assert abs(slope - want) <= 64 * U * (scale * 10), (j, slope, want)


@pytest.mark.parametrize("T,D,dtype", [(64, 4096, "bf16"), (20000, 40, "f16")])
def test_a_run_of_them_behind_a_routing(T, D, dtype):
    """route -> sort -> dispatch -> experts -> combine and back, in a graph on a stream of its own,
    replayed with other queries; each expert multiplies by its own number."""
    E, k = 24, 4
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s, dt=F32: torch.zeros(s, dtype=dt, device="cuda")
    logits, x, scale = new(T, E), new(T, D, dt=DT[dtype]), 0.5 + torch.rand((E,), generator=g, device="cuda")
    idx, weight, load = new(T, k, dt=I32), new(T, k), new(E, dt=I32)
    offsets, source, place = new(E + 1, dt=I32), new(T * k, dt=I32), new(T, k, dt=I32)
    rows, out, g_out = new(T * k, D, dt=DT[dtype]), new(T, D, dt=DT[dtype]), new(T, D, dt=DT[dtype])
    g_rows, g_weight, dx, dlogits = new(T * k, D, dt=DT[dtype]), new(T, k), new(T, D, dt=DT[dtype]), new(T, E)

    def step():
        bt.boute_route(logits, None, 0, 1, 1, 1, True, 1.0, idx, weight, load)
        bt.boute_expert_sort(idx, offsets, source, place)
        bt.boute_expert_dispatch(x, place, rows)
        of = torch.searchsorted(offsets, torch.arange(T * k, dtype=I32, device="cuda"), right=True) - 1
        by = scale[of.clamp(max=E - 1)][:, None]
        rows.copy_(rows * by)
        bt.boute_expert_combine(rows, place, weight, out)
        bt.boute_expert_combine_grad(g_out, rows, place, weight, g_rows, g_weight)
        g_rows.copy_(g_rows * by)
        bt.boute_expert_dispatch_grad(g_rows, place, dx)
        bt.boute_route_grad(logits, 0, True, 1.0, idx, g_weight, dlogits)

    def fill():
        for a in (logits, x, g_out):
            a.copy_(torch.randn(a.shape, generator=g, device="cuda"))

    fill()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for _ in range(2):
            fill()
            graph.replay()
    s.synchronize()
    assert torch.equal(offsets.diff(), load) and offsets[E] == T * k
    p = torch.softmax(logits.double(), 1)
    i64 = idx.long()
    w = torch.gather(p, 1, i64)
    w /= w.sum(1, keepdim=True)
    sc = scale.double()[i64]
    want = (w * sc).sum(1, keepdim=True) * x.double()
    # three roundings to the type (of the rows, times their number, and the sum), positive weights
    tol = 3.5 * EPS[dtype] * (w * sc).sum(1, keepdim=True) * x.double().abs() + 4 * TINY[dtype] + 1e-6
    assert ((out.double() - want).abs() <= tol).all()
    want = (w * sc).sum(1, keepdim=True) * g_out.double()
    tol = 3.5 * EPS[dtype] * (w * sc).sum(1, keepdim=True) * g_out.double().abs() + 4 * TINY[dtype] + 1e-6
    assert ((dx.double() - want).abs() <= tol).all()
    dots = (g_out.double() * x.double()).sum(1, keepdim=True) * sc
    size = (g_out.double() * x.double()).abs().sum(1, keepdim=True) * sc
    assert ((g_weight.double() - dots).abs() <= (1.01 * EPS[dtype] + (D / 8 + 16) * U) * size).all()


def test_streams_of_their_own():
    T, k, E, D = 3000, 4, 50, 64
    x = torch.randn((T, D), device="cuda")
    idx = torch.from_numpy(choices(8, T, k, E, none=0)).cuda()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    rows, out = torch.zeros((T * k, D), device="cuda"), torch.zeros((T, D), device="cuda")
    w = torch.full((T, k), 0.25, device="cuda")
    torch.cuda.synchronize()
    _, _, place = sort(idx, E, s)
    bt.boute_expert_dispatch(x, place, rows, s)
    bt.boute_expert_combine(rows, place, w, out, s)
    s.synchronize()
    assert torch.equal(out, x)


def test_offsets_beyond_32_bits():
    """Rows whose elements lie beyond 2^32: the last places of a long array."""
    D, k = 1 << 16, 1
    R = (1 << 32) // D + 40
    rows = torch.zeros((R, D), dtype=torch.bfloat16, device="cuda")
    T = 50
    place = torch.arange(R - T, R, dtype=I32, device="cuda").view(T, k)
    x = torch.randn((T, D), device="cuda").bfloat16()
    bt.boute_expert_dispatch(x, place, rows)
    assert torch.equal(rows[R - T:], x) and not rows[:R - T].any()
    out = torch.empty_like(x)
    bt.boute_expert_combine(rows, place, torch.ones((T, k), device="cuda"), out)
    assert torch.equal(out, x)
    g_weight = torch.empty((T, k), device="cuda")
    bt.boute_expert_combine_grad(x, rows, place, torch.ones((T, k), device="cuda"), rows, g_weight)
    assert torch.equal(rows[R - T:], x)
    want = (x.double() ** 2).sum(1)
    assert ((g_weight[:, 0].double() - want).abs() <= (D / 8 + 16) * U * want).all()
