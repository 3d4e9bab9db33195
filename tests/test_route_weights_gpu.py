"""Weights of the routing are rounded to fp32 once, whatever the rule."""
import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from oracle import block

pytestmark = pytest.mark.gpu


# 64-bit arithmetic throughout, so half a step of fp32 and next to nothing on top (2^-40: some hundred roundings of 2^-53, and arguments of up
# to 2^9 in exponentials)
@pytest.mark.parametrize("score,groups", [("softmax", 1), ("softmax", 4), ("sigmoid", 1), ("sigmoid", 4)])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 4, 1), (64, 128, 8), (1001, 8, 2), (300, 512, 10)])
def test_one_rounding(tokens, experts, top_k, bias, renormalise, score, groups):
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, experts, generator=g) * 3
    b = 0.05 * torch.randn(experts, generator=g) if bias else None
    rule = dict(score=score, groups=groups, top_groups=max(1, groups // 2), renormalise=renormalise)
    if groups > 1:
        top_k = min(top_k, experts // groups * rule["top_groups"])
    ids, w, _ = bd.route(x.cuda(), top_k, bias=None if b is None else b.cuda(), **rule)
    ri, rw = block.route(x.double().numpy(), top_k, bias=None if b is None else b.double().numpy(), **rule)
    assert np.array_equal(ids.cpu().numpy(), ri)
    assert (np.abs(w.double().cpu().numpy() - rw) <= (2.0 ** -24 + 2.0 ** -40) * np.abs(rw) + 2.0 ** -149).all()
    bd.poll_status()


def test_a_bias_of_zeros_changes_nothing():
    for experts in (8, 60, 128, 512):
        x = torch.randn(700, experts, generator=torch.Generator().manual_seed(experts)).cuda()
        for score in ("softmax", "sigmoid"):
            for renormalise in (False, True):
                a = bd.route(x, 4, score=score, renormalise=renormalise, plan=False)
                b = bd.route(x, 4, score=score, renormalise=renormalise, bias=torch.zeros(experts, device="cuda"), plan=False)
                if score == "softmax":                            # (sigmoids of different logits can be equal: other numbers first)
                    assert torch.equal(a[0], b[0])
                same = (a[0] == b[0]).all(1)
                assert torch.equal(a[1][same], b[1][same]) and same.float().mean() > 0.9
