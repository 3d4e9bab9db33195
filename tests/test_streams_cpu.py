"""Calls with a `stream` allocate on that stream: shown with a library, an allocator and streams that only write down what happens."""
import contextlib
import types

import pytest
import torch

from paper_2501_01144_b200 import binding


class Recorder:
    """Which stream is current at each allocation and each call of the library."""

    def __init__(self, monkeypatch):
        self.now, self.seen = 0, []
        empty = torch.empty
        monkeypatch.setattr(torch, "empty", lambda *a, **k: (self.seen.append(("memory", self.now)), empty(*a, **k))[1])
        monkeypatch.setattr(binding, "_current_stream", lambda: self.now, raising=False)
        monkeypatch.setattr(torch.cuda, "stream", self.switch)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw: types.SimpleNamespace(cuda_stream=raw))
        monkeypatch.setattr(binding, "_stream", lambda stream=None: self.now if stream is None else stream.cuda_stream)

    @contextlib.contextmanager
    def switch(self, stream):
        before, self.now = self.now, stream.cuda_stream
        try:
            yield
        finally:
            self.now = before


SIDE = types.SimpleNamespace(cuda_stream=5)


@pytest.mark.parametrize("gated", [False, True])
def test_quantised_experts_are_allocated_on_the_calls_stream(gated, monkeypatch):
    log = Recorder(monkeypatch)

    class Weights:
        def __init__(self, experts, rows, K, device):
            torch.empty(1)
            self.experts, self.rows, self.K = experts, rows, K

        def expert(self, e):
            return self

    monkeypatch.setattr(binding, "ExpertWeights", Weights)
    monkeypatch.setattr(binding, "quantize_weights", lambda W, select, out=None: log.seen.append(("kernel", log.now)))
    W = torch.zeros(2, 64, 32)
    binding.quantize_experts(W, gated=gated, stream=SIDE)
    assert log.seen == [("memory", 5), ("kernel", 5), ("kernel", 5)] and log.now == 0
    log.seen.clear()
    binding.quantize_experts(W, gated=gated)
    assert log.seen == [("memory", 0), ("kernel", 0), ("kernel", 0)]
