"""Plain products, many tiles per cluster, give the same bits every time, within the products' bound of the sums in 64 bits (the epilogue's
stores beside the main loop's shared-memory loads)."""
import pytest
import torch

import paper_2501_01144_b200 as bd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", [(2048, 28672, 1024), (512, 28672, 4096), (300, 14336, 512), (4096, 8192, 256)])
def test_plain_products_repeat(M, N, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(M)
    W = bd.quantize_weights(torch.randn(N, K, generator=g, device="cuda") * K ** -0.5, bd.SELECT_TWO_STAGE)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    out = torch.empty(M, N, dtype=dtype, device="cuda")
    first = bd.linear(x, W, dtype=dtype)
    for _ in range(30):
        assert torch.equal(bd.linear(x, W, out=out), first)
    xq, wq = bd.dequantize(bd.quantize_act(x)).double(), bd.dequantize(W).double()
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for at in range(0, N, 4096):
        want, size = xq @ wq[at:at + 4096].T, xq.abs() @ wq[at:at + 4096].abs().T
        assert ((first[:, at:at + 4096].double() - want).abs() <= 1e-6 * size + half * (want.abs() + 1e-6 * size)).all()
    bd.poll_status()
