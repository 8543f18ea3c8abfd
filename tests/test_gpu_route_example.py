"""The operators together, as examples/route_queries.py uses them: scores of answers, a router
trained through their gradients, and its bias searched by the optimisation loop; and the debug
build's bounds checks over small and ragged cases of each operator (in a child process)."""
import importlib.util
import os
import subprocess
import sys
import textwrap

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def example():
    path = os.path.join(ROOT, "examples", "route_queries.py")
    spec = importlib.util.spec_from_file_location("route_queries", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_training_and_search():
    ex = example()
    r = ex.main(queries=600, vocabulary=1000, steps=40, evaluations=14)
    assert r["losses"][-1] < r["losses"][0]
    assert bool(torch.isfinite(r["g_logits"].float()).all()) and float(r["g_logits"].float().norm()) > 0
    Y = r["search"]["Y"]
    assert len(Y) == 14 and np.isfinite(Y).all() and len(r["front"]) >= 1


def test_gradient_through_the_whole_path_against_differences():
    """The logits' gradient through scores and router against central differences of the same path
    computed in 64 bits, for a few logits of one answer (k is all replicas: the choice is fixed)."""
    ex = example()
    a = ex.Answers(queries=12, vocabulary=40, seed=3)
    a.logits = a.logits.float()
    a.offsets = a.offsets.clone()
    router = ex.Router(a.scores())
    x = router.logits(a.scores())
    idx, w, _ = router.route(x, x.shape[1])
    loss_of = ex.errors(router, a, idx)
    dx = torch.empty_like(x)
    ex.bt.boute_route_grad(x, ex.bt.BOUTE_ROUTE_SOFTMAX, True, 1.0, idx, loss_of.contiguous(), dx)
    g = a.backward(((dx @ router.W.t())[:, :4] / router.std).contiguous())

    weak = torch.tensor(ex.WEAKNESS, dtype=torch.float64).repeat_interleave(router.replicas)
    off, t = a.offsets.tolist(), a.targets.cpu()

    def loss(z):
        lp = torch.log_softmax(z, 1)
        H = -(lp.exp() * lp).sum(1)
        lp = lp[torch.arange(len(t)), t]
        total = 0.0
        for q in range(len(off) - 1):
            s = slice(off[q], off[q + 1])
            f = torch.stack([lp[s].mean(), lp[s].min(), H[s].mean(), H[s].max()])
            f = (f - router.mean.double().cpu()) / router.std.double().cpu()
            p = torch.softmax(torch.cat([f, torch.ones(1, dtype=torch.float64)]) @
                              router.W.double().cpu(), 0)
            total = total + (p * weak).sum() * a.difficulty.double().cpu()[q]
        return float(total)

    z = a.logits.double().cpu()
    for row, col in ((0, 3), (5, int(t[5])), (off[4], 17), (off[7] + 1, int(t[off[7] + 1]))):
        step = torch.zeros_like(z)
        step[row, col] = 1e-5
        want = (loss(z + step) - loss(z - step)) / 2e-5
        # fp32 all along: a few units of the largest gradient's rounding
        assert abs(float(g[row, col]) - want) <= 1e-5 * max(1.0, float(g.abs().max()))


CHILD = textwrap.dedent(r"""
    import sys
    sys.path.insert(0, ROOT); sys.path.insert(0, HERE)
    from paper_2602_10729_gb300 import boute as bt, build as bld
    bt.load(bld.build(debug=True))
    import torch
    import test_gpu_answers as ta, test_gpu_routing as tr

    def report(what):
        r = bt.boute_bounds_report()
        if r is not None:
            print(what, f"VIOLATION unit={r[0]} line={r[1]} index={r[2]} extent={r[3]}")
        return r is None

    ok = True
    for T, V, k, dt in [(1, 1, 1, "f32"), (3, 33, 32, "bf16"), (2, 5003, 20, "f16"),
                        (1, 131072, 32, "bf16"), (40, 40001, 17, "f32")]:
        ta.test_forward_sizes_types_and_places(dt, T, V, k, 1.25, 1, 1)
        ok &= report(f"forward {T} {V}")
    ta.test_alternatives_with_ties(20011, 32)
    ok &= report("ties")
    for name in ("tiny", "mixed", "one-among-many", "long"):
        ta.test_scores_of_answers(name, True)
        ta.test_gradient_of_the_scores(name, False)
        ok &= report(name)
    for shape in ((5, 7, 1, 1, 1, 3), (70, 192, 8, 4, 2, 6), (6, 1024, 16, 3, 2, 32)):
        tr.test_route_sizes_and_types(tr.SIG, "bf16", *shape)
        ok &= report(f"route {shape}")
    print("BOUNDS_OK" if ok else "BOUNDS_BAD")
""")


def test_bounds_checked_build():
    code = f"ROOT = {ROOT!r}; HERE = {HERE!r}\n" + CHILD
    p = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=900,
                       cwd=ROOT)
    assert p.returncode == 0, p.stdout + p.stderr
    assert "BOUNDS_OK" in p.stdout, p.stdout
