"""Calls of host threads on problems of different sizes at the same time: a kernel's limit of shared
memory is the process's."""
import threading

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [(1000, 560), (1000, 520, 800)])
def test_box_decompositions_of_different_capacities(sizes):
    """13 (n + 2) doubles each; fronts of five points."""
    failed, results = [], {}

    def work(n):
        try:
            torch.cuda.set_device(0)
            f64 = dict(dtype=torch.float64, device="cuda")
            front = torch.zeros((1, n, 3), **f64)
            front[0, :5] = torch.tensor([[1, 5, 3], [2, 4, 1], [3, 3, 4], [4, 2, 2], [5, 1, 5.0]], **f64)
            P = torch.tensor([5], dtype=torch.int32, device="cuda")
            ref = torch.zeros((1, 3), **f64)
            lo, hi = (torch.zeros((1, 2 * n + 2, 3), device="cuda") for _ in range(2))
            K = torch.zeros((1,), dtype=torch.int32, device="cuda")
            stream = torch.cuda.Stream()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                for i in range(3000):
                    bt.boute_box_decompose(front, P, 1, n, 3, ref, lo, hi, K)
                    if i % 100 == 99:
                        stream.synchronize()
            results[n] = int(K[0]), lo[0, :int(K[0])].cpu(), hi[0, :int(K[0])].cpu()
        except Exception as error:
            failed.append((n, error))

    threads = [threading.Thread(target=work, args=(n,)) for n in sizes]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert failed == []
    first = results[sizes[0]]
    assert first[0] > 0
    for k, lo, hi in results.values():
        assert k == first[0] and torch.equal(lo, first[1]) and torch.equal(hi, first[2])
