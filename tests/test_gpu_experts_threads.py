"""Calls of host threads that sort among different numbers of experts at the same time."""
import threading

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt
from test_gpu_experts import check_sort, choices

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,k,counts", [(4000, 4, (1024, 760)), (400000, 2, (512, 256)),
                                        (400000, 2, (1024, 300))])
def test_threads_with_different_numbers_of_experts(T, k, counts):
    """No call fails, and all give what they give alone."""
    failed, results = [], {}

    def work(E):
        try:
            torch.cuda.set_device(0)
            idx = torch.from_numpy(choices(T, T, k, E, twice=True)).cuda()
            new = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")
            out = new(E + 1), new(T * k), new(T, k)
            stream = torch.cuda.Stream()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                for i in range(3000):
                    bt.boute_expert_sort(idx, *out)
                    if i % 100 == 99:
                        stream.synchronize()
            results[E] = idx, out
        except Exception as error:
            failed.append((E, error))

    threads = [threading.Thread(target=work, args=(E,)) for E in counts]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert failed == []
    torch.cuda.synchronize()
    for E, (idx, out) in results.items():
        check_sort(idx.cpu().numpy(), E)
        alone = [torch.empty_like(x) for x in out]
        bt.boute_expert_sort(idx, *alone)
        assert all(torch.equal(a, b) for a, b in zip(out, alone))
