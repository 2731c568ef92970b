"""A stream of another device than the current one is refused: the kernels would run there,
on memory of this one."""
import pytest
import torch

from paper_2110_02861_amd import bq


class Stream:
    """A stand-in for torch.cuda.Stream, which needs a GPU."""

    def __init__(self, device_index):
        self.device_index = device_index
        self.cuda_stream = 0


def test_stream_of_another_device(monkeypatch):
    current = Stream(1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: current)
    assert bq._other(None) is None and bq._other(current) is None
    side = Stream(1)
    assert bq._other(side) is side
    with pytest.raises(ValueError, match="cuda:0"):
        bq._other(Stream(0))
