"""The activation far below zero, where it is tiny but the product with the other half is not."""
import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from oracle import block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 300])                      # narrow items, and items of 256 tokens
def test_gates_far_below_zero(tokens):
    gates = [-3.0, -20.0, -60.0, -80.0, -84.0, -88.0, -92.0, -96.0]   # one per block of 32 channels
    inter, hidden = 32 * len(gates), 32
    W = torch.zeros(1, 2 * inter, hidden)
    W[0, :inter, 0] = torch.tensor(gates).repeat_interleave(32)
    W[0, inter:, 1] = 2.0 ** 100
    up = bd.quantize_experts(W.cuda(), gated=True)
    down = bd.quantize_experts(torch.zeros(1, 8, inter).cuda())
    x = torch.zeros(tokens, hidden, device="cuda")
    x[:, :2] = 1.0
    plan = bd.expert_plan(torch.zeros(tokens, 1, dtype=torch.int32, device="cuda"), 1)
    inner = torch.empty(tokens, 1, inter, device="cuda")
    bd.expert_mlp(x, plan, torch.ones(tokens, 1, device="cuda"), up, down, inner=inner)
    bd.poll_status()
    rows = bd.dequantize(up.expert(0)).double().cpu().numpy()[np.argsort(block.gated_order(inter))]
    xq = bd.dequantize(bd.quantize_act(x)).double().cpu().numpy()[0]
    g, u = rows[:inter] @ xq, rows[inter:] @ xq
    assert g.min() < -90 and u.min() > 2.0 ** 99
    h = block.activate(g, "silu") * u
    # a block of equal values is off by half a step of its grid, 1/16 at most; the exponential is a multiple of 2^-149 where it is no normal number
    off = np.abs(g * u) * 2.0 ** -149
    assert (np.abs(inner[:, 0].double().cpu().numpy() - h) <= (1 / 16 + 2.0 ** -16) * np.abs(h) + 2 * off).all()
