"""What the block calls' binding refuses or does without, shown without a GPU."""
import types

import pytest
import torch

from paper_2501_01144_b200 import binding


@pytest.mark.parametrize("rows,K", [(256, 4096), (128, 4096), (4096, 128), (127, 4096)])
def test_a_quantised_norm_refuses_an_operand_of_another_shape(rows, K, monkeypatch):
    # [4096, 256] and [256, 4096] have buffers of the same sizes: only the shape tells them apart
    got = []
    monkeypatch.setattr(binding, "_block", types.SimpleNamespace(norm=lambda *a: got.append(a[14]) or (None, None, *a[14])))
    q = binding.QTensor.from_buffers(*(torch.zeros(1, dtype=torch.uint8) for _ in range(3)), rows, K)
    y = torch.zeros(4096, 256)
    with pytest.raises(ValueError, match="out_n"):
        binding.residual_norm(y, torch.ones(256), quantise=True, out_n=q)
    assert not got
    same = binding.QTensor.from_buffers(q.codes, q.ids, q.scales, 4096, 256)
    assert binding.residual_norm(y, torch.ones(256), quantise=True, out_n=same)[1] is same and got == [(q.codes, q.ids, q.scales)]


def test_dequantize_needs_the_library_alone(monkeypatch, tmp_path):
    calls = []
    monkeypatch.setattr(binding, "_block", None)
    monkeypatch.setattr(binding, "_BLOCK_PATH", str(tmp_path / "_block.so"))
    monkeypatch.setattr(binding, "load", lambda: types.SimpleNamespace(bd_dequantize=lambda *a: calls.append(a) or 0))
    monkeypatch.setattr(binding, "_stream", lambda stream=None: 0)
    q = binding.QTensor.from_buffers(*(torch.zeros(64, dtype=torch.uint8) for _ in range(3)), 2, 64)
    assert binding.dequantize(q).shape == (2, 64) and len(calls) == 1
