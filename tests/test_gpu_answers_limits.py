"""The operators over a model's answers where their inputs or launches are at a limit, against plain
64-bit forms."""
import numpy as np
import pytest
import torch

from _answers import U, answer_grad, answer_rows
from paper_2602_10729_gb300 import boute as bt
from test_gpu_answers import answers, check_forward, close, forward, logits, scored

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
