"""The experts' parts are added up in fp32: a bf16 result is the fp32 one rounded once, whatever the workspace has room for."""
import ctypes

import pytest
import torch

import paper_2501_01144_b200 as bd

pytestmark = pytest.mark.gpu


def step(tokens, experts, top_k, hidden, inter, n):
    g = torch.Generator(device="cuda").manual_seed(tokens + n)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    up = bd.quantize_experts(r(experts, 2 * inter, hidden) * hidden ** -0.5, bd.SELECT_TWO_STAGE, gated=True)
    down = bd.quantize_experts(r(experts, n, inter) * inter ** -0.5, bd.SELECT_TWO_STAGE)
    _, w, plan = bd.route(r(tokens, experts), top_k)
    return r(tokens, hidden).bfloat16(), plan, w, up, down


# narrow items and items of 256 tokens; outputs of one tile and several, odd numbers of chunks, widths that no pass over the columns divides
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inter,n", [(1, 8, 4, 256, 128, 256), (5, 4, 2, 96, 32, 8), (70, 8, 3, 32, 64, 40), (300, 6, 2, 224, 96, 520), (1000, 4, 2, 128, 160, 264), (900, 3, 2, 32, 96, 1032)])
def test_a_bf16_result_is_the_fp32_one_rounded_once(tokens, experts, top_k, hidden, inter, n):
    args = step(tokens, experts, top_k, hidden, inter, n)
    want = bd.expert_mlp(*args, dtype=torch.float32)
    assert torch.equal(bd.expert_mlp(*args), want.bfloat16())
    # the least workspace (fewer columns at a time), its contents of no account, and one between the two sizes
    n_bytes, full = ctypes.c_size_t(), bd.expert_mlp_workspace_size(tokens, top_k, *args[3:])
    assert bd.load().bd_expert_mlp_workspace_size(ctypes.c_int64(tokens), ctypes.c_int64(top_k), *(ctypes.c_char_p(w._c) for w in args[3:]), bd.BF16, ctypes.byref(n_bytes)) == 0
    least = n_bytes.value
    assert least <= full == bd.expert_mlp_workspace_size(tokens, top_k, *args[3:], torch.float32)
    for size in (least, (least + full) // 2, full):
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        wide = torch.full((tokens, n + 16), 3.0, dtype=torch.bfloat16, device="cuda")
        bd.expert_mlp(*args, out=wide[:, 8:n + 8], workspace=ws)
        assert torch.equal(wide[:, 8:n + 8], want.bfloat16())
        assert (wide[:, :8] == 3).all() and (wide[:, n + 8:] == 3).all()
    bd.poll_status()
