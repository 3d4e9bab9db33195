"""More experts than a warp has lanes, and more than there are items of one round: the schedule's scan goes on over groups of 32."""
import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from test_experts_gpu import check, ids_by_counts, tokens_of, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,experts,top_k", [(1, 33, 3), (40, 64, 8), (200, 100, 4), (130, 512, 2), (5, 512, 32), (2100, 40, 2)])
def test_more_than_32_experts(tokens, experts, top_k):
    up, down = weights(experts, 96, 64, 136)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    ids = torch.topk(torch.rand(tokens, experts, generator=g, device="cuda"), top_k)[1].to(torch.int32)
    x, w = tokens_of(tokens, 96, torch.bfloat16), torch.rand(tokens, top_k, generator=g, device="cuda")
    check(x, ids, w, up, down)
    check(x, ids, w, up, down, "gelu", torch.bfloat16)


@pytest.mark.parametrize("where", [[31, 32], [0, 63, 64, 99], [40], [32, 33, 34, 95, 96]])
def test_experts_without_tokens_in_between(where):
    counts = np.zeros(100, int)
    counts[where] = [1 + 130 * (k % 3) + k for k in range(len(where))]
    up, down = weights(100, 64, 32, 72)
    ids = ids_by_counts(counts, 2, 400)
    assert torch.equal(bd.expert_plan(ids, 100).count.cpu().long(), torch.from_numpy(counts))
    check(tokens_of(400, 64, torch.bfloat16), ids, torch.rand(400, 2, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda"), up, down)
