"""The norm that a step of AdamW is clipped by lies on the context's device: its
address is read and written there."""
import pytest
import torch


class Library:
    calls = 0

    def tlc_adamw(self, *args):
        self.calls += 1
        self.result = args[-1]
        return 0


class Buffer:
    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index


class Result:
    def __init__(self, index):
        self.buffer, self.ptr = Buffer(index), 64


class Weights:
    """What adamw() asks of its list."""
    device = torch.device("cuda", 1)
    count, args, grad_args, state_args, clock_ptr = 0, (None,) * 3, (None,) * 2, (0,) * 5, 8

    def lay_out_options(self, *rates):
        return None


def test_a_result_of_another_device_is_refused(monkeypatch):
    from paper_1802_07389_amd import tlc
    library = Library()
    monkeypatch.setattr(tlc, "lib", library)
    ctx = object.__new__(tlc.TrainContext)
    ctx.handle, ctx.index = None, 1
    for index in (0, 2, -1):  # -1: host memory
        with pytest.raises(ValueError, match="device"):
            ctx.adamw(Weights(), 0.1, max_norm=1.0, result=Result(index))
    assert library.calls == 0
    ctx.adamw(Weights(), 0.1, max_norm=1.0, result=Result(1))
    assert library.calls == 1 and library.result == 64
    ctx.adamw(Weights(), 0.1)
    assert library.calls == 2 and library.result is None
