"""The binding of the calls over a model's answers launches on the current device alone: tensors or
streams of another are refused. (On tensors that say where they are, and a library that notes its
calls.)"""
import types

import pytest
import torch

from paper_2602_10729_gb300 import boute as bt

F32, I32, I64 = torch.float32, torch.int32, torch.int64


class On:
    """What the binding asks of a tensor, on device `dev`."""

    def __init__(self, dev, dtype, *shape):
        self.dev, self.dtype, self.shape, self.is_cuda = dev, dtype, shape, dev >= 0

    def stride(self):
        return (self.shape[1], 1)

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.dev

    def data_ptr(self):
        return 4096


def calls(dev):
    """(function, arguments) of each call with tensors on device dev[i]."""
    at = iter(dev)
    t = lambda *a: On(next(at), *a)
    return [
        (bt.boute_token_logprobs, lambda: (t(F32, 4, 9), t(I64, 4), 1.0, t(F32, 4), t(F32, 4), t(F32, 4),
                                           t(I64, 4, 2), t(F32, 4, 2))),
        (bt.boute_token_logprobs_grad, lambda: (t(F32, 4, 9), t(I64, 4), 1.0, t(F32, 4), t(F32, 4),
                                                t(F32, 4), t(F32, 4), t(F32, 4, 9))),
        (bt.boute_answer_scores, lambda: (t(F32, 4), t(F32, 4), t(I64, 4), t(I64, 3), t(F32, 2, 4),
                                          t(I32, 2))),
        (bt.boute_answer_scores_grad, lambda: (t(F32, 4), t(F32, 4), t(I64, 4), t(I64, 3), t(F32, 2, 4),
                                               t(F32, 4), t(F32, 4))),
        (bt.boute_route, lambda: (t(F32, 4, 9), t(F32, 9), 0, 1, 1, 1, True, 1.0, t(I32, 4, 2),
                                  t(F32, 4, 2), t(I32, 9))),
        (bt.boute_route_grad, lambda: (t(F32, 4, 9), 0, True, 1.0, t(I32, 4, 2), t(F32, 4, 2),
                                       t(F32, 4, 9))),
    ]


TENSORS = (7, 7, 6, 7, 5, 4)  # of each call


@pytest.fixture
def launched(monkeypatch):
    done = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: done.append((name, a[-1])) or 0

    monkeypatch.setattr(bt, "load", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(bt, "_raw_stream", lambda dev: 1000 + dev)
    return done


@pytest.mark.parametrize("call", range(6))
def test_tensors_of_one_device_that_is_not_the_current_one(call, launched):
    f, args = calls([1] * 8)[call]
    with pytest.raises(ValueError):
        f(*args())
    assert launched == []


@pytest.mark.parametrize("call", range(6))
def test_one_tensor_of_another_device(call, launched):
    for other in (1, -1):
        for i in range(TENSORS[call]):
            f, args = calls([other if i == j else 0 for j in range(8)])[call]
            with pytest.raises(ValueError):
                f(*args())
    assert launched == []


@pytest.mark.parametrize("call", range(6))
def test_the_current_device_and_its_streams(call, launched):
    f, args = calls([0] * 8)[call]
    f(*args())
    f, args = calls([0] * 8)[call]
    f(*args(), stream=types.SimpleNamespace(cuda_stream=77, device_index=0))
    f, args = calls([0] * 8)[call]
    f(*args(), stream=55)
    assert [s for _, s in launched] == [1000, 77, 55]
    f, args = calls([0] * 8)[call]
    with pytest.raises(ValueError):
        f(*args(), stream=types.SimpleNamespace(cuda_stream=77, device_index=1))
    assert len(launched) == 3
