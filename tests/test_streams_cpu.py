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


def operand(rows=4, K=32):
    return binding.QTensor.from_buffers(*(torch.zeros(64, dtype=torch.uint8) for _ in range(3)), rows, K)


def cache():
    c = binding.KVCache.__new__(binding.KVCache)
    c.capacity, c.head_dim, c.k, c.v, c._ws = 32, 32, operand(32), operand(32), None
    c._c = binding._CKVCache(c.k.c_struct(), c.v.c_struct(), None, 0, 32, 32, 4)
    return c


X, P = torch.zeros(4, 32), torch.zeros(2, 4)
CALLS = {
    "quantize_weights": lambda **s: binding.quantize_weights(X, **s), "quantize_act": lambda **s: binding.quantize_act(X, **s), "quantize_bs": lambda **s: binding.quantize_bs(X, 32, **s),
    "gemm": lambda **s: binding.gemm(operand(), operand(), **s), "gemm_batched": lambda **s: binding.gemm_batched([operand()], [operand()], **s), "gemm_requant": lambda **s: binding.gemm_requant(operand(), operand(), **s),
    "linear": lambda **s: binding.linear(X, operand(), **s), "linear_requant": lambda **s: binding.linear_requant(X, operand(), **s), "linear_bs": lambda **s: binding.linear_bs(X, operand(), 32, **s),
    "attention": lambda **s: binding.attention([operand()], [operand()], [operand()], dump=True, **s), "export_canonical": lambda **s: binding.export_canonical(operand(), **s),
    "export_canonical_bs": lambda **s: binding.export_canonical_bs(operand(), 32, **s), "import_canonical": lambda **s: binding.import_canonical(*(torch.zeros(4, n, dtype=torch.uint8) for n in (16, 1, 1)), **s),
    "dequantize": lambda **s: binding.dequantize(operand(), **s), "scores": lambda **s: cache().scores(operand(), **s), "pv": lambda **s: cache().pv(P, **s),
    "kvcache_scores_batched": lambda **s: binding.kvcache_scores_batched([cache()], [operand()], **s), "kvcache_pv_batched": lambda **s: binding.kvcache_pv_batched([cache()], P[None], **s),
    "kvcache_attention": lambda **s: binding.kvcache_attention([cache()], [operand()], 1.0, **s)}


@pytest.mark.parametrize("name", CALLS)
def test_results_and_workspaces_are_allocated_on_the_calls_stream(name, monkeypatch):
    log = Recorder(monkeypatch)

    class Library:
        def __getattr__(self, call):
            def fake(*a):
                if call.endswith("_size") or call.endswith("_sizes"):
                    for b in a[-(3 if call.endswith("s") else 1):]:
                        b._obj.value = 64
                else:
                    log.seen.append(("kernel", log.now))
                return 0
            return fake

    monkeypatch.setattr(binding, "load", Library)
    monkeypatch.setattr(binding, "_load_block", lambda: types.SimpleNamespace(dequantize=lambda *a: None))
    monkeypatch.setattr(binding, "_block", None)
    monkeypatch.setattr(binding, "_src", lambda x: (x.data_ptr(), 0, x.stride(0)))
    for stream, args in ((5, dict(stream=SIDE)), (0, {})):
        log.seen.clear()
        CALLS[name](**args)
        assert {what for what, _ in log.seen} == {"memory", "kernel"} and {at for _, at in log.seen} == {stream} and log.now == 0
