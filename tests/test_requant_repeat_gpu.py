"""Products with the requantising epilogue, many tiles per cluster, give the same bits every time (its scattered stores beside the main
loop's shared-memory loads)."""
import pytest
import torch

import paper_2501_01144_b200 as bd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(2048, 28672, 1024), (512, 28672, 4096), (300, 14336, 512)])
def test_requantised_products_repeat(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M)
    W = bd.quantize_weights(torch.randn(N, K, generator=g, device="cuda") * K ** -0.5, bd.SELECT_TWO_STAGE)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    first = bd.linear_requant(x, W)
    for _ in range(10):
        q = bd.linear_requant(x, W)
        assert torch.equal(q.codes, first.codes) and torch.equal(q.ids, first.ids) and torch.equal(q.scales, first.scales)
    want = bd.quantize_act(bd.linear(x, W, dtype=torch.float32))
    assert torch.equal(first.codes, want.codes)
    bd.poll_status()
