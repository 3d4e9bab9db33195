"""The experts' gated products on the GPU: the requantised values between the products against 64 bits, block by block, and the
result against the second product of exactly those values."""
import numpy as np
import pytest
import torch

import oracle
import paper_2501_01144_b200 as bd
from oracle import block

pytestmark = pytest.mark.gpu


def weights(experts, hidden, inter, n, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    up = bd.quantize_experts(r(experts, 2 * inter, hidden) * hidden ** -0.5, bd.SELECT_TWO_STAGE, gated=True)
    down = bd.quantize_experts(r(experts, n, inter) * inter ** -0.5, bd.SELECT_TWO_STAGE)
    return up, down


def tokens_of(tokens, hidden, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(tokens, hidden, generator=g, device="cuda") * torch.where(torch.rand(hidden, generator=g, device="cuda") < 0.02, 10.0, 1.0)).to(dtype)


def ids_by_counts(counts, top_k, tokens, seed=2):
    """ids [tokens, top_k] with expert e in counts[e] tokens, -1 elsewhere."""
    rng = np.random.default_rng(seed)
    ids = np.full((tokens, top_k), -1, np.int32)
    for e in np.argsort(-np.asarray(counts), kind="stable"):
        free = np.nonzero((ids < 0).any(1))[0]
        for t in rng.permutation(free)[: counts[e]]:
            ids[t, np.nonzero(ids[t] < 0)[0][0]] = e
    return torch.from_numpy(ids).cuda()


def check(x, ids, w, up, down, act="silu", dtype=torch.float32, out=None, workspace=None):
    tokens, k = ids.shape
    inter, n = down.K, down.rows
    plan = bd.expert_plan(ids, up.experts)
    inner = torch.full((tokens, k, inter), 7.0, device="cuda")
    y = bd.expert_mlp(x, plan, w, up, down, activation=act, dtype=dtype, inner=inner, out=out, workspace=workspace)
    assert torch.equal(y, bd.expert_mlp(x, plan, w, up, down, activation=act, dtype=dtype))
    bd.poll_status()
    xq = bd.dequantize(bd.quantize_act(x)).double()
    got, yw, total = inner.double(), torch.zeros(tokens, n, dtype=torch.float64, device="cuda"), torch.zeros(tokens, n, dtype=torch.float64, device="cuda")
    parts = torch.zeros_like(yw)
    blocks = unclear = 0
    order = torch.from_numpy(np.argsort(block.gated_order(inter))).cuda()
    for e in range(up.experts):
        token, slot = torch.nonzero(ids == e, as_tuple=True)
        if not token.numel():
            continue
        W = bd.dequantize(up.expert(e)).double()[order]
        gate, upper = xq[token] @ W[:inter].T, xq[token] @ W[inter:].T
        sums = xq[token].abs() @ W.abs().T                        # sum of |x| |w|: the products' error is 2^-22 of it at most here
        a = torch.from_numpy(block.activate(gate.cpu().numpy(), act)).cuda()
        h = a * upper
        slope = 1.13                                              # the steepest that either activation gets
        eps = 2.0 ** -22 * (slope * sums[:, :inter] * upper.abs() + a.abs() * sums[:, inter:]) + 2.0 ** -19 * upper.abs() * (a.abs() + (1 + gate.abs() if act == "gelu" else 0) * 2.0 ** -3) + 1e-30
        # every decision of the quantiser is one on floor(4 |h| / 2^e): where no element of a block is near a multiple of 2^(e - 2),
        # the block's values are those of the 64-bit ones
        hb, eb, mine = (z.unflatten(-1, (-1, 32)) for z in (h, eps, got[token, slot]))
        top = hb.abs().amax(-1, keepdim=True)
        unit = torch.exp2(torch.floor(torch.log2(top.clamp(min=1e-300))) - 4)
        near = (hb.abs() / unit - torch.round(hb.abs() / unit)).abs() * unit <= eb
        clear = ~((near & (torch.round(hb.abs() / unit) > 0)).any(-1)) & (top[..., 0] > 2.0 ** -100)
        want = oracle.dequantize(*oracle.quantize(h.float().cpu().numpy()))
        same = (mine == torch.from_numpy(want).cuda().unflatten(-1, (-1, 32))).all(-1)
        assert (same | ~clear).all(), f"expert {e}: {int((~same & clear).sum())} blocks differ"
        assert ((mine - hb).abs() <= 2 * 4 * unit + eb).all()     # gaps of the grids: at most 6 half units = 3 * 2^e, half of that
        blocks, unclear = blocks + clear.numel(), unclear + int((~clear).sum())
        D = bd.dequantize(down.expert(e)).double()
        part = (got[token, slot] @ D.T) * w[token, slot].double()[:, None]
        yw.index_add_(0, token, part)
        parts.index_add_(0, token, part.abs())
        total.index_add_(0, token, (got[token, slot].abs() @ D.abs().T) * w[token, slot].double().abs()[:, None])
    assert unclear <= 0.2 * blocks + 40
    assert (got[ids < 0] == 0).all()
    # products within 1e-6 of the sum of magnitudes; k products and sums in fp32; bf16: a rounding of each part and one of the result
    tol = 1e-6 * total + (k + 2) * 2.0 ** -24 * parts
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * parts + 2.0 ** -8 * (yw.abs() + 2.0 ** -8 * parts)
    assert ((y.double() - yw).abs() <= tol + 1e-30).all()
    return y


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inter,n,act", [
    (1, 8, 2, 256, 128, 256, "silu"), (7, 4, 4, 96, 32, 8, "gelu"), (64, 16, 4, 512, 160, 264, "silu"), (300, 6, 2, 224, 96, 512, "gelu"), (1, 1, 1, 32, 32, 40, "silu")])
def test_against_64_bits(tokens, experts, top_k, hidden, inter, n, act, dtype):
    up, down = weights(experts, hidden, inter, n)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.stack([torch.randperm(experts, generator=g, device="cuda")[:top_k] for _ in range(tokens)]).to(torch.int32)
    w = torch.rand(tokens, top_k, generator=g, device="cuda")
    x = tokens_of(tokens, hidden, dtype)
    for ydtype in (torch.float32, torch.bfloat16):
        check(x, ids, w, up, down, act, ydtype)


@pytest.mark.parametrize("counts", [[256, 0, 1], [257, 16, 17, 0], [0, 0, 0, 5], [15, 31, 33, 63, 65, 127, 128, 129], [600, 1, 300], [512, 512]])
def test_tokens_of_every_number_per_expert(counts):
    tokens = max(max(counts), 260)
    ids = ids_by_counts(counts, len(counts), tokens)
    assert torch.equal(bd.expert_plan(ids, len(counts)).count.cpu(), torch.tensor(counts, dtype=torch.int32))
    up, down = weights(len(counts), 256, 96, 320)
    w = torch.rand(tokens, len(counts), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") - 0.3
    check(tokens_of(tokens, 256, torch.bfloat16), ids, w, up, down, dtype=torch.bfloat16)


@pytest.mark.parametrize("tokens,hidden,inter,n", [(700, 1024, 4096, 1024), (300, 256, 8192, 4096)])
def test_many_items_for_every_cluster(tokens, hidden, inter, n):
    up, down = weights(2, hidden, inter, n)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, 2, (tokens, 1), generator=g, device="cuda", dtype=torch.int32)
    x, w = tokens_of(tokens, hidden, torch.bfloat16), torch.rand(tokens, 1, generator=g, device="cuda")
    y = check(x, ids, w, up, down)
    plan = bd.expert_plan(ids, 2)
    for _ in range(8):
        assert torch.equal(bd.expert_mlp(x, plan, w, up, down, dtype=torch.float32), y)


def test_sizes_of_a_model():
    up, down = weights(8, 2048, 1408, 2048)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.topk(torch.rand(200, 8, generator=g, device="cuda"), 3)[1].to(torch.int32)
    check(tokens_of(200, 2048, torch.bfloat16), ids, torch.rand(200, 3, generator=g, device="cuda"), up, down, dtype=torch.bfloat16)


def test_routed_and_normed_block_as_a_model_runs_it():
    hidden, inter, experts, k = 512, 256, 12, 3
    up, down = weights(experts, hidden, inter, hidden)
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    router, w1, w2, post = r(experts, hidden) * 0.05, 1 + 0.1 * r(hidden), 1 + 0.1 * r(hidden), 1 + 0.1 * r(hidden)
    for tokens in (1, 33, 200):
        residual, branch = (r(tokens, hidden) * 2).bfloat16(), r(tokens, hidden).bfloat16()
        h, n = bd.residual_norm(branch, w1.bfloat16(), residual)
        ids, w, plan = bd.route(n.float() @ router.T, k, score="sigmoid", scale=2.0)
        y = bd.expert_mlp(n, plan, w, up, down)
        h2, q = bd.residual_norm(y, w2.bfloat16(), h, post_weight=post.bfloat16(), quantise=True)
        bd.poll_status()
        assert torch.equal(y, check(n, ids, w, up, down, dtype=torch.bfloat16))
        y64, h64 = y.double().cpu().numpy(), h.double().cpu().numpy()
        want = h64 + block.norm(y64, post.bfloat16().double().cpu().numpy(), None, False, 1e-6, 0.0)
        assert (np.abs(h2.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * np.abs(want - h64) + 2.0 ** -20 * np.abs(h64) + 1e-30).all()
        assert torch.equal(q.codes, bd.quantize_act(bd.residual_norm(y, w2.bfloat16(), h, post_weight=post.bfloat16())[1]).codes)


def test_a_token_does_not_depend_on_the_others_nor_on_the_call():
    up, down = weights(5, 320, 64, 128)
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w = tokens_of(400, 320, torch.bfloat16), torch.rand(400, 2, generator=g, device="cuda")
    ids = torch.stack([torch.randperm(5, generator=g, device="cuda")[:2] for _ in range(400)]).to(torch.int32)
    whole = bd.expert_mlp(x, bd.expert_plan(ids, 5), w, up, down)
    for at, to in ((0, 1), (1, 40), (17, 300)):
        part = ids[at:to].contiguous()
        assert torch.equal(bd.expert_mlp(x[at:to], bd.expert_plan(part, 5), w[at:to], up, down), whole[at:to])


def test_empty_rows_repeated_experts_strides_and_given_buffers():
    up, down = weights(4, 128, 64, 72)
    ids = torch.tensor([[1, 1, 3], [-1, -1, -1], [-1, 2, -1], [0, 1, 2], [3, 3, 3]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[0.5, 0.25, 1.0], [1, 1, 1], [1, 2, 3], [0, -1, 1], [0.1, 0.2, 0.3]], device="cuda")
    wide = torch.full((5, 160), float("nan"), dtype=torch.bfloat16, device="cuda")
    x = wide[:, 16:144]
    x.copy_(tokens_of(5, 128, torch.bfloat16))
    out = torch.full((5, 100), 3.0, device="cuda")
    need = bd.expert_mlp_workspace_size(5, 3, up, down, torch.float32)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    y = check(x, ids, w, up, down, out=out[:, 8:80], workspace=ws)
    assert y.data_ptr() == out[:, 8:80].data_ptr() and (y[1] == 0).all()
    assert (out[:, :8] == 3).all() and (out[:, 80:] == 3).all()
    none = bd.expert_mlp(x[:0], bd.expert_plan(ids[:0], 4), w[:0], up, down)
    assert none.shape == (0, 72)


def test_captured_calls_follow_their_inputs():
    up, down = weights(6, 256, 128, 256)
    g = torch.Generator(device="cuda").manual_seed(8)
    x, logits = tokens_of(96, 256, torch.bfloat16), torch.randn(96, 6, generator=g, device="cuda")
    valid = torch.tensor([96], dtype=torch.int32, device="cuda")

    def step():
        ids, w, plan = bd.route(logits, 2, valid=valid)
        return ids, w, bd.expert_mlp(x, plan, w, up, down)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ids, w, y = step()
    for n in (96, 3, 0, 50):
        logits.copy_(torch.randn(96, 6, generator=g, device="cuda"))
        x.copy_(tokens_of(96, 256, torch.bfloat16, seed=n))
        valid.fill_(n)
        graph.replay()
        got = y.clone()
        assert torch.equal(got, step()[2]) and (got[n:] == 0).all()
        if n:
            assert torch.equal(got[:n], check(x[:n], ids[:n].contiguous(), w[:n].contiguous(), up, down, dtype=torch.bfloat16))
    bd.poll_status()


def test_plans_change_from_call_to_call_in_the_same_memory():
    up, down = weights(24, 512, 256, 512)
    g = torch.Generator(device="cuda").manual_seed(12)
    x, w = tokens_of(64, 512, torch.bfloat16), torch.rand(64, 4, generator=g, device="cuda")
    every = [torch.topk(torch.rand(64, 24, generator=g, device="cuda") + 3 * (torch.arange(24, device="cuda") % (k + 2) == 0), 4)[1].to(torch.int32) for k in range(6)]
    plan = bd.expert_plan(every[0], 24)
    want = []
    for ids in every:
        torch.cuda.synchronize()
        want.append(bd.expert_mlp(x, bd.expert_plan(ids, 24), w, up, down))
        torch.cuda.synchronize()
    got = []
    for _ in range(20):                                           # one plan's memory, written again right before each call
        for ids in every:
            got.append(bd.expert_mlp(x, bd.expert_plan(ids, 24, out=plan), w, up, down))
    bd.poll_status()
    assert all(torch.equal(y, want[k % 6]) for k, y in enumerate(got))


def test_calls_on_two_streams():
    up, down = weights(6, 512, 256, 512)
    g = torch.Generator(device="cuda").manual_seed(9)
    jobs = []
    for n in (40, 300):
        ids = torch.topk(torch.rand(n, 6, generator=g, device="cuda"), 2)[1].to(torch.int32)
        jobs.append((tokens_of(n, 512, torch.bfloat16, n), ids, torch.rand(n, 2, generator=g, device="cuda")))
    want = [bd.expert_mlp(x, bd.expert_plan(i, 6), w, up, down) for x, i, w in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    got = [[] for _ in jobs]
    for _ in range(10):
        for k, (x, i, w) in enumerate(jobs):
            got[k].append(bd.expert_mlp(x, bd.expert_plan(i, 6, stream=streams[k]), w, up, down, stream=streams[k]))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(y, want[k]) for y in got[k])


def test_what_is_not_finite_is_told_and_stays_in_its_token():
    up, down = weights(3, 128, 64, 128)
    x, ids = tokens_of(20, 128, torch.float32), torch.arange(20, device="cuda").remainder(3).to(torch.int32)[:, None].contiguous()
    w = torch.ones(20, 1, device="cuda")
    want = bd.expert_mlp(x, bd.expert_plan(ids, 3), w, up, down)
    x[4, 7] = torch.nan
    y = bd.expert_mlp(x, bd.expert_plan(ids, 3), w, up, down)
    with pytest.raises(bd.BdError) as e:
        bd.poll_status()
    assert e.value.status == 6
    keep = torch.arange(20, device="cuda") != 4
    assert torch.equal(y[keep], want[keep])


def test_a_plan_out_of_its_bounds_is_told_and_addresses_nothing():
    up, down = weights(3, 128, 64, 128)
    x, ids = tokens_of(20, 128, torch.float32), torch.arange(20, device="cuda").remainder(3).to(torch.int32)[:, None].contiguous()
    w = torch.ones(20, 1, device="cuda")
    want = bd.expert_mlp(x, bd.expert_plan(ids, 3), w, up, down)
    for name, at, value in (("count", 1, 2 ** 30), ("count", 1, -5), ("start", 1, 2 ** 31 - 128), ("start", 1, 64), ("start", 1, -128)):
        plan = bd.expert_plan(ids, 3)
        getattr(plan, name)[at] = value
        y = bd.expert_mlp(x, plan, w, up, down)
        with pytest.raises(bd.BdError) as e:
            bd.poll_status()
        assert e.value.status == 10
        keep = ids[:, 0] != 1
        assert torch.equal(y[keep], want[keep])
    plan = bd.expert_plan(ids, 3)
    plan.place[5] = 2 ** 31 - 1
    y = bd.expert_mlp(x, plan, w, up, down)
    with pytest.raises(bd.BdError) as e:
        bd.poll_status()
    assert e.value.status == 10
    keep = torch.arange(20, device="cuda") != 5
    assert torch.equal(y[keep], want[keep]) and (y[5] == 0).all()


@pytest.mark.parametrize("tokens, count", [(20, 21), (20, 100), (3, 128), (200, 201), (200, 256)])
def test_a_plan_with_more_rows_than_tokens_is_told(tokens, count):
    # inside the padded operand, but more than an expert can have: the copies of a call's tokens are sized by their number
    up, down = weights(2, 128, 64, 128)
    x, ids = tokens_of(tokens, 128, torch.bfloat16), torch.arange(tokens, device="cuda").remainder(2).to(torch.int32)[:, None].contiguous()
    w = torch.ones(tokens, 1, device="cuda")
    want = bd.expert_mlp(x, bd.expert_plan(ids, 2), w, up, down)
    plan = bd.expert_plan(ids, 2)
    plan.count[0] = count
    y = bd.expert_mlp(x, plan, w, up, down)
    with pytest.raises(bd.BdError) as e:
        bd.poll_status()
    assert e.value.status == 10
    assert torch.equal(y[1::2], want[1::2])


def test_experts_are_operands_of_their_own():
    w = torch.randn(3, 128, 96, generator=torch.Generator().manual_seed(1)).cuda()
    e = bd.quantize_experts(w, gated=True)
    order = torch.from_numpy(block.gated_order(64))
    for k in range(3):
        q = bd.quantize_weights(w[k][order].contiguous())
        assert all(torch.equal(a, b) for a, b in zip((q.codes, q.ids, q.scales), (e.codes[k], e.ids[k], e.scales[k])))
    x = tokens_of(5, 96, torch.bfloat16)
    assert torch.equal(bd.linear(x, e.expert(1)), bd.linear(x, bd.quantize_weights(w[1][order].contiguous())))


@pytest.mark.parametrize("tokens", [4, 600])                      # narrow items, and items of 256 tokens
def test_a_wait_that_runs_out_is_told_and_the_next_call_is_served(tokens):
    up, down = weights(2, 512, 256, 256)
    ids = torch.randint(0, 2, (tokens, 1), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    x, w, plan = tokens_of(tokens, 512, torch.bfloat16), torch.ones(tokens, 1, device="cuda"), bd.expert_plan(ids, 2)
    good = bd.expert_mlp(x, plan, w, up, down)
    bd.poll_status()
    try:
        # the first copy of packed weights of every CTA is never started: nothing is in flight for it, and the wait for it ends
        bd.debug_fault(poll_limit=10 * 1024, skip_first_code_stage=True)
        bd.expert_mlp(x, plan, w, up, down)
        with pytest.raises(bd.BdError) as e:
            bd.poll_status()
        assert e.value.status == 7
    finally:
        bd.debug_fault(0, False)
    for _ in range(3):
        assert torch.equal(bd.expert_mlp(x, plan, w, up, down), good)
    bd.poll_status()


def test_two_plans_and_two_workspaces_in_two_graphs():
    up, down = weights(6, 256, 128, 256)
    g = torch.Generator(device="cuda").manual_seed(21)
    jobs = []
    for n in (48, 200):
        x, logits = tokens_of(n, 256, torch.bfloat16, n), torch.randn(n, 6, generator=g, device="cuda")
        ws = torch.empty(bd.expert_mlp_workspace_size(n, 2, up, down), dtype=torch.uint8, device="cuda")

        def step(x=x, logits=logits, ws=ws):
            ids, w, plan = bd.route(logits, 2)
            return bd.expert_mlp(x, plan, w, up, down, workspace=ws)

        want = step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = step()
        jobs.append((graph, y, want, x, logits, ws))                  # a graph does not keep its inputs alive
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (graph, *_) in zip(streams, jobs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    bd.poll_status()
    for _, y, want, *_ in jobs:
        assert torch.equal(y, want)


def test_experts_of_large_and_tiny_scales():
    g = torch.Generator(device="cuda").manual_seed(22)
    for gain in (2.0 ** -40, 2.0 ** 20):
        W = torch.randn(2, 128, 128, generator=g, device="cuda") * 128 ** -0.5
        up = bd.quantize_experts(W, bd.SELECT_TWO_STAGE, gated=True)
        down = bd.quantize_experts(torch.randn(2, 72, 64, generator=g, device="cuda") * gain, bd.SELECT_TWO_STAGE)
        ids = torch.arange(30, device="cuda").remainder(2).to(torch.int32)[:, None].contiguous()
        check(tokens_of(30, 128, torch.float32), ids, torch.ones(30, 1, device="cuda"), up, down)
