"""The calls over experts' rows and hidden states at their limits: the bounds-checked build, arrays
beyond 2^32 elements, a workspace that graphs share, a run of all of them."""
import os
import subprocess
import sys
import textwrap

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from test_gpu_hidden import EPS, STEP, Plain, backward, forward, inputs

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
CHILD = textwrap.dedent(r"""
    import sys
    sys.path.insert(0, ROOT); sys.path.insert(0, HERE)
    from paper_2602_10729_gb300 import boute as bt, build as bld
    bt.load(bld.build(debug=True))
    import test_gpu_experts as te, test_gpu_hidden as th

    def report(what):
        r = bt.boute_bounds_report()
        print(what, "ok" if r is None else f"VIOLATION {r}")
        return r is None

    ok = True
    for T, k, E in ((0, 2, 5), (1, 8, 8), (513, 8, 61), (4099, 6, 61), (4097, 8, 1024), (32769, 1, 7),
                    (100003, 5, 257), (300000, 4, 2)):
        te.check_sort(te.choices(T, T, k, E, twice=T > 50000), E)
        ok &= report(f"sort {T} {k} {E}")
    for row in te.ROWS:
        te.test_dispatch_and_its_gradient(*row)
        te.test_combine_and_its_gradient(*row)
        ok &= report(f"rows {row}")
    for size in th.SIZES:
        th.test_forward(*size)
        th.test_gradient(*size)
        ok &= report(f"hidden {size}")
    th.test_positions_of_several_passes(8200)
    th.check_grad(8192, 16448, 32, "bf16", 1.0)
    ok &= report("passes and pieces")
    print("ALL_CLEAN" if ok else "FOUND_VIOLATIONS")
""")


def test_no_index_outside_its_extent():
    code = f"ROOT = {os.path.dirname(HERE)!r}\nHERE = {HERE!r}\n" + CHILD
    res = subprocess.run([sys.executable, "-c", code], cwd=HERE, capture_output=True, text=True,
                         timeout=1500)
    assert res.returncode == 0, (res.stdout + res.stderr)[-4000:]
    assert "ALL_CLEAN" in res.stdout, res.stdout[-4000:]


def test_a_weight_beyond_32_bits():
    """131072 + 100 tokens of 32768 elements: 2^32 elements and more, 8.6 GB. Zero but for a few
    tokens, the last ones among them, so that everything is known: the logits of the others are 0."""
    T, V, D = 3, 131072 + 100, 32768
    w = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    h = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda")
    h[:, -1], h[:, 0] = 1.0, torch.tensor([0.5, 1.0, 2.0])
    at = torch.tensor([5, 70000, 131071, 131072, V - 1], device="cuda")
    w[at, -1] = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0], dtype=torch.bfloat16, device="cuda")
    w[at, 0] = 1.0
    t = torch.tensor([V - 1, 131072, 17], device="cuda")
    z = (h[:, -1:].double() * w[at, -1].double() + h[:, :1].double() * w[at, 0].double())
    s = torch.exp(z).sum(1) + (V - len(at))
    lse = torch.log(s)
    lp, H, got = forward(h, w, t, 1.0)
    assert ((got.double() - lse).abs() < 1e-5).all()
    want = torch.stack([z[0, 4], z[1, 3], z[2, 0] * 0]) - lse
    assert ((lp.double() - want).abs() < 1e-5).all()
    g = torch.tensor([1.0, -2.0, 0.5], device="cuda")
    dh, dw = backward(h, w, t, 1.0, lse.float(), None, g, None)
    p = torch.exp(z - lse[:, None])
    c = -p * g.double()[:, None]
    c[0, 4] += 1.0
    c[1, 3] -= 2.0
    want = c.t() @ h.double()
    size = c.abs().t() @ h.double().abs()
    tol = 3 * EPS["bf16"] * size + 1e-6
    assert ((dw[at].double() - want).abs() <= tol).all()
    # a token that is a target with logit 0, and one that is not
    q = torch.exp(-lse)
    want = ((-q * g.double())[:, None] * h.double()).sum(0)
    near = lambda a, b: ((a.double() - b).abs() <= 3 * EPS["bf16"] * (q * g.double().abs()).sum() * 4 + 1e-7)
    assert near(dw[131070], want).all()
    assert ((dw[17].double() - want - 0.5 * h[2].double()).abs() <= 2 * EPS["bf16"] * 1.1).all()
    want = c @ w[at].double()
    tol = 3 * EPS["bf16"] * (c.abs() @ w[at].double().abs()) + 1e-6
    assert ((dh.double() - want).abs() <= tol).all()


def test_two_graphs_share_a_workspace():
    """Captured calls of different sizes and kinds over one workspace, replayed in turn on a stream."""
    a, b = inputs(300, 2000, 128, "bf16"), inputs(40, 5000, 64, "f16", seed=3)
    n = max(bt.boute_hidden_logprobs_workspace(*x[:2], grad) for x in (a, b) for grad in (False, True))
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    plain = [Plain(*x, 1.0) for x in (a, b)]
    outs = [[torch.zeros((x[0].shape[0],), device="cuda") for _ in range(3)] for x in (a, b)]
    grads = [[torch.zeros_like(y) for y in x[:2]] for x in (a, b)]
    g = [torch.full((x[0].shape[0],), 0.1, device="cuda") for x in (a, b)]
    graphs = []
    for x, o, d, gi in zip((a, b), outs, grads, g):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                bt.boute_hidden_logprobs(*x, 1.0, *o, ws)
                bt.boute_hidden_logprobs_grad(*x, 1.0, o[2], o[1], gi, gi, *d, ws)
            graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(2):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for x, o, p, d, gi, dt in zip((a, b), outs, plain, grads, g, ("bf16", "f16")):
        p.check(*o)
        p.lse, p.H = o[2].double(), o[1].double()
        dh, dw, th, tw = p.grad(gi, gi, dt)
        assert ((d[0].double() - dh).abs() <= th).all() and ((d[1].double() - dw).abs() <= tw).all()


def test_a_layer_of_experts_to_the_answers_scores_and_back():
    """All of them as a model's step has them: hidden states routed, sorted, sent to experts (a factor
    each), brought back, their answers' log-probabilities and scores, and the way back to the hidden
    states; differences along a direction agree with the gradient."""
    T, D, E, k, V = 260, 64, 12, 3, 700
    gen = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")
    f16, i32 = torch.float16, torch.int32
    x0 = rand(T, D)
    wr, wv = rand(E, D) * 0.2, (rand(V, D) * 0.2).half()
    by = 0.5 + torch.rand((E,), generator=gen, device="cuda")
    t = torch.randint(0, V, (T,), generator=gen, device="cuda")
    off = torch.tensor([0, 100, 180, T], dtype=torch.int64, device="cuda")
    gs = rand(3, 4) * torch.tensor([1.0, 0.0, 1.0, 0.0], device="cuda")  # (means: smooth)
    new = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device="cuda")
    idx, weight, place, source = new(T, k, dt=i32), new(T, k), new(T, k, dt=i32), new(T * k, dt=i32)
    offsets, ws = new(E + 1, dt=i32), None

    def expert_of():
        r = torch.arange(T * k, dtype=i32, device="cuda")
        return (torch.searchsorted(offsets, r, right=True) - 1).clamp(max=E - 1)

    def step(x, fixed=False):
        """(sum of gs times scores, what the backward pass needs); fixed: the choices of before."""
        logits = x @ wr.t()
        if not fixed:
            bt.boute_route(logits, None, 0, 1, 1, 1, True, 1.0, idx, weight)
            bt.boute_expert_sort(idx, offsets, source, place)
        else:
            p = torch.softmax(logits, 1).gather(1, idx.long())
            weight.copy_(p / p.sum(1, keepdim=True))
        rows, sent, out = new(T * k, D), new(T * k, D), new(T, D)
        bt.boute_expert_dispatch(x, place, rows)
        sent = rows * by[expert_of()][:, None]
        bt.boute_expert_combine(sent, place, weight, out)
        h = out.half()
        lp, H, lse = new(T), new(T), new(T)
        w = torch.empty((max(bt.boute_hidden_logprobs_workspace(h, wv, b) for b in (0, 1)),),
                        dtype=torch.uint8, device="cuda")
        bt.boute_hidden_logprobs(h, wv, t, 1.0, lp, H, lse, w)
        scores, counts = new(3, 4), new(3, dt=i32)
        bt.boute_answer_scores(lp, H, t, off, scores, counts)
        return (scores.double() * gs.double()).sum().item(), (logits, sent, h, lp, H, lse, w)

    f0, (logits, sent, h, lp, H, lse, w) = step(x0)
    gl, gh = new(T), new(T)
    bt.boute_answer_scores_grad(lp, H, t, off, gs, gl, gh)
    dh, dwv = torch.empty_like(h), torch.empty_like(wv)
    bt.boute_hidden_logprobs_grad(h, wv, t, 1.0, lse, H, gl, gh, dh, dwv, w)
    g_sent, g_weight, dx, dlogits = new(T * k, D), new(T, k), new(T, D), new(T, E)
    bt.boute_expert_combine_grad(dh.float(), sent, place, weight, g_sent, g_weight)
    bt.boute_expert_dispatch_grad(g_sent * by[expert_of()][:, None], place, dx)
    bt.boute_route_grad(logits, 0, True, 1.0, idx, g_weight, dlogits)
    dx = dx.double() + (dlogits @ wr).double()
    # the states are rounded to fp16 on the way (2^-11 of each, random): a difference over 2 eps is off
    # by some 2^-11 |dh . h| / sqrt(T D) a side; a direction along the gradient, where it is largest
    d = (dx / dx.norm()).float()
    eps = 2.0
    up, _ = step(x0 + eps * d, True)
    down, _ = step(x0 - eps * d, True)
    slope, want = (up - down) / (2 * eps), dx.norm().item()
    noise = 2.0 ** -11 * (dh.double() * h.double()).norm().item() / eps * 8
    curve = 0.05 * want  # (the third derivative over steps of 2 / sqrt(T D) = 0.016 an element)
    assert abs(slope - want) <= noise + curve, (slope, want, noise)
