"""The operators over a model's answers on both sides of the sizes where another kernel, or another
spread of the work, takes over, against plain 64-bit forms. Tolerances as in the other tests."""
import numpy as np
import pytest
import torch

from _answers import U, answer_grad, answer_rows
from paper_2602_10729_gb300 import boute as bt
from test_gpu_answers import DT, answers, check_forward, check_grad, close, forward, scored
from test_gpu_routing import SIG, SOFT, check_many, queries

pytestmark = pytest.mark.gpu

SMS = 152


# Experts 64, 128, 256, 512; choices 4, 8; 64 queries (one block, with a load); 16 and 24 queries an SM
@pytest.mark.parametrize("E", [64, 65, 128, 129, 256, 257, 512, 513])
@pytest.mark.parametrize("mode,dtype,bias", [(SOFT, "bf16", False), (SIG, "f32", True)])
def test_routing_where_kernels_change(E, mode, dtype, bias):
    x = queries(E, 19, E, dtype, 0.7)
    x[3, ::2] = -float("inf")
    x[7] = 0.25
    g = torch.Generator().manual_seed(E)
    b = (torch.randint(-100, 100, (E,), generator=g).float() * 1e-3).cuda() if bias else None
    most = (16 if E <= 128 else 24) * SMS
    for k in (4, 5, 8, 9):
        for T in (64, 65, most - 1, most):
            check_many(x, b, mode, 1, 1, 1, k, True, 1.0, T=T)


def tiled(x, T):
    return x[torch.arange(T) % len(x)].cuda()


# Rows in clusters of 8, 4 and 2 blocks and in one; of 4, 2 and 1 warps where rows are many and short
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,k", [(SMS, 40000, 20), (SMS + 1, 40000, 20), (2 * SMS, 40000, 8),
                                   (2 * SMS + 1, 40000, 8), (4 * SMS, 20000, 9), (4 * SMS + 1, 20000, 9),
                                   (48 * SMS - 1, 1500, 8), (48 * SMS, 1500, 8), (48 * SMS, 1500, 9),
                                   (76, 32767, 5), (77, 32767, 5)])
def test_log_probabilities_where_the_spread_changes(dtype, T, V, k):
    g = torch.Generator().manual_seed(T + k)
    x = (torch.randn((17, V), generator=g) * 3).to(DT[dtype])
    x[2, V // 2:] = -float("inf")
    t = torch.randint(0, V // 2, (17,), generator=g)
    xs, ts = tiled(x, T), tiled(t, T)
    out = forward(xs, ts, 1.25, k)
    at = torch.cat([torch.arange(17), torch.arange(T - 17, T)])  # the first rows and the last
    check_forward(x[at % 17], t[at % 17], 1.25, k, tuple(v[at.cuda()] for v in out))
    rows = (torch.arange(T) % 17).cuda()
    assert torch.equal(out[3], out[3][:17][rows])
    gl, gh = torch.randn(17, generator=g), torch.randn(17, generator=g)
    dx = torch.empty_like(xs)
    bt.boute_token_logprobs_grad(xs, ts, 1.25, out[2], out[1], tiled(gl, T), tiled(gh, T), dx)
    check_grad(x[at % 17], t[at % 17], 1.25, gl[at % 17], gh[at % 17], dx[at.cuda()], dtype)
    if V % 8 == 0:  # (rows that lie alike against 16-byte boundaries have their sums in one order)
        assert all(torch.equal(v, v[:17][rows]) for v in (*out, dx))


# Teams of 8 and 32 lanes, a block, clusters of 2, 4 and 8, by the mean length and the answers' number
@pytest.mark.parametrize("Q,mean", [(100, 24), (100, 25), (60, 512), (60, 513), (40, 1024), (40, 1025),
                                    (40, 2049), (40, 4097), (304, 2049), (305, 2049), (608, 1025),
                                    (609, 1025)])
def test_scores_where_teams_change(Q, mean):
    g = torch.Generator().manual_seed(Q + mean)
    n = torch.randint(0, 2 * mean, (Q - 1,), generator=g)
    n = (n.double() * (mean * (Q - 1)) / n.sum()).long()
    lengths = n.tolist() + [Q * mean - int(n.sum())]
    lp, ent, t, off = answers(Q, lengths)
    got, cnt = scored(lp, ent, t, off)
    want, n = answer_rows(lp.numpy(), ent.numpy(), t.numpy(), off.numpy())
    assert cnt.tolist() == n.tolist()
    assert np.array_equal(got[:, [1, 3]], want[:, [1, 3]].astype(np.float32))
    close(got[:, [0, 2]], want[:, [0, 2]], U * 8 * (4 + 4 * np.sqrt(np.maximum(n, 1)))[:, None])
    gs = torch.randn((Q, 4), generator=g)
    gl, gh = torch.full_like(lp, 9.0).cuda(), torch.full_like(lp, 9.0).cuda()
    bt.boute_answer_scores_grad(lp.cuda(), ent.cuda(), t.cuda(), off.cuda(), gs.cuda(), gl, gh)
    wl, wh = answer_grad(lp.numpy(), ent.numpy(), t.numpy(), off.numpy(), gs.double().numpy())
    close(gl.cpu().numpy(), wl, 4 * U * 10)
    close(gh.cpu().numpy(), wh, 4 * U * 10)
