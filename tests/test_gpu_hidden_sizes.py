"""Log-probabilities from hidden states where the kernels' layouts change: positions in columns whose
reduction is summed in parts, by one group of warps and by two, one tile of positions and several, at
any alignment; gradients whose sums are in parts; and the bounds-checked build on all of them."""
import os
import subprocess
import sys
import textwrap

import pytest

from test_gpu_hidden import check_grad, test_forward as forward_holds

pytestmark = pytest.mark.gpu

SIZES = [  # T, V, D, dtype, scale, pitch, shift
    (33, 3000, 513, "bf16", 1.0, 0, 0), (40, 3000, 520, "f16", 1.0, 0, 0),
    (64, 3000, 1030, "bf16", 1.25, 0, 0), (64, 700, 1024, "f16", 1.0, 8, 8),
    (65, 3000, 1100, "f16", 1.0, 0, 0), (96, 1025, 1032, "bf16", 1.0, 0, 0),
    (130, 3000, 2048, "bf16", 1.0 / 0.7, 0, 0), (128, 2000, 4096, "f16", 1.0, 0, 0),
    (170, 1001, 1536, "f16", 1.0, 3, 5), (170, 1001, 1536, "bf16", 1.0, 0, 0),
    (300, 2000, 2000, "bf16", 1.0, 0, 0), (341, 511, 1025, "f16", 1.0, 1, 1)]


@pytest.mark.parametrize("size", SIZES)
def test_forward(size):
    forward_holds(*size)


@pytest.mark.parametrize("size", SIZES)
def test_gradient(size):
    check_grad(*size, ent=size[0] % 2 == 0)


# many positions, and many tokens of a piece beside a large hidden size, in two pieces
LONG = [(20000, 300, 40, "f16", 1.0, 0, 0), (20000, 300, 41, "f16", 1.0, 1, 3),
        (140000, 300, 33, "bf16", 1.0, 0, 0), (5000, 27000, 2048, "f16", 1.0, 0, 0)]


@pytest.mark.parametrize("size", LONG)
def test_gradient_of_long_sums(size):
    check_grad(*size)


CHILD = textwrap.dedent(r"""
    import sys
    sys.path.insert(0, ROOT); sys.path.insert(0, HERE)
    from paper_2602_10729_gb300 import boute as bt, build as bld
    bt.load(bld.build(debug=True))
    import test_gpu_hidden as th, test_gpu_hidden_sizes as ts, test_gpu_hidden_far as tf

    ok = True
    def report(what):
        global ok
        r = bt.boute_bounds_report()
        print(what, "ok" if r is None else f"VIOLATION {r}")
        ok &= r is None

    for size in ts.SIZES:
        ts.test_forward(size)
        ts.test_gradient(size)
        report(size)
    for T, V, D in ((20, 1000, 64), (130, 2000, 64), (600, 513, 32)):
        tf.test_gradient_of_far_logits("f16", T, V, D, 1.25, 512.0)
        report((T, V, D))
    for size in ts.LONG[:3]:
        ts.test_gradient_of_long_sums(size)
        report(size)
    tf.test_far_positions_of_several_passes()
    report("passes")
    print("ALL_CLEAN" if ok else "FOUND_VIOLATIONS")
""")


def test_no_index_outside_its_extent():
    here = os.path.dirname(os.path.abspath(__file__))
    code = f"ROOT = {os.path.dirname(here)!r}\nHERE = {here!r}\n" + CHILD
    res = subprocess.run([sys.executable, "-c", code], cwd=here, capture_output=True, text=True,
                         timeout=1500)
    assert res.returncode == 0, (res.stdout + res.stderr)[-4000:]
    assert "ALL_CLEAN" in res.stdout, res.stdout[-4000:]
