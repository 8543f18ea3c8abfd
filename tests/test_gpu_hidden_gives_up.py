"""What the gradient of hidden states writes once one of its launches has given up a wait. The word
that says so is set by hand in the workspace of a captured call, whose launches before the
coefficients' (which clear it) are taken out of the graph: what they leave is there from a call
before."""
import ctypes

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from test_gpu_hidden import inputs

pytestmark = pytest.mark.gpu

TIMEOUT = 6  # BOUTE_ERR_TIMEOUT


def chain(graph):
    """The nodes of a graph that is one chain, in order."""
    cu = ctypes.CDLL("libcuda.so.1")
    n, node = ctypes.c_size_t(1), ctypes.c_void_p()
    assert cu.cuGraphGetRootNodes(graph, ctypes.byref(node), ctypes.byref(n)) == 0 and n.value == 1
    nodes, edge = [], ctypes.c_uint64()
    while True:
        nodes.append(node)
        n, after = ctypes.c_size_t(1), ctypes.c_void_p()
        assert cu.cuGraphNodeGetDependentNodes_v2(node, ctypes.byref(after), ctypes.byref(edge),
                                                  ctypes.byref(n)) == 0
        if n.value == 0 or not after.value:
            return cu, nodes
        node = after


@pytest.mark.parametrize("T,dtype,pieces", [(20, "f16", 1), (100, "bf16", 1), (300, "bf16", 1),
                                            (8192, "bf16", 2)])
def test_no_wrong_number_is_written_after_a_wait_that_gave_up(T, dtype, pieces):
    V = 16384 + 300 if pieces == 2 else 700
    h, w, t = inputs(T, V, 64, dtype)
    lp, H, lse = (torch.zeros((T,), device="cuda") for _ in range(3))
    g = torch.ones((T,), device="cuda")
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    ws = torch.zeros((max(bt.boute_hidden_logprobs_workspace(h, w, b) for b in (False, True)),),
                     dtype=torch.uint8, device="cuda")
    bt.boute_hidden_logprobs(h, w, t, 1.0, lp, H, lse, ws)
    step = lambda: bt.boute_hidden_logprobs_grad(h, w, t, 1.0, lse, H, g, g, dh, dw, ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            step()
    cu, nodes = chain(ctypes.c_void_p(graph.raw_cuda_graph()))
    own = 2 * pieces + 1  # (the coefficients and the products of each piece, dh's sums)
    assert len(nodes) > own
    for node in nodes[:-own]:
        assert cu.cuGraphDestroyNode(node) == 0
    graph.instantiate()
    status = ws[:4].view(torch.int32)
    for value in (0, TIMEOUT):
        want = dh.clone(), dw.clone()
        dh.fill_(7), dw.fill_(7)
        status.fill_(value)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if value == 0:
            assert torch.equal(dh, want[0]) and torch.equal(dw, want[1])
        else:
            assert dh.isnan().all() and dw.isnan().all()
