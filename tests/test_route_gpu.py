"""Routing to experts and the plan of their rows on the GPU, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from oracle import block

pytestmark = pytest.mark.gpu

F32_STEP = 2.0 ** -24


def logits_of(tokens, experts, dtype, seed, spread=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(tokens, experts, generator=g) * spread + 0.5 * torch.randn(experts, generator=g)).to(dtype)


def check(x, top_k, plan=True, bias=None, valid=None, **rule):
    """x on the CPU; returns what the call gave."""
    dev = x.cuda()
    ids, w, p = bd.route(dev, top_k, bias=None if bias is None else bias.cuda(), valid=None if valid is None else torch.tensor([valid], dtype=torch.int32, device="cuda"), plan=plan, **rule)
    ri, rw = block.route(x.double().numpy(), top_k, bias=None if bias is None else bias.double().numpy(), valid=valid, **rule)
    assert ids.dtype == torch.int32 and w.dtype == torch.float32
    assert np.array_equal(ids.cpu().numpy(), ri)
    # one rounding to fp32; a softmax that is not renormalised divides by a sum of fp32 exponentials (two steps each, and their
    # argument's step times its size, at most exp(-d) d < 1) added in at most 16 + 5 additions
    tol = 2 * F32_STEP if rule.get("renormalise", True) or rule.get("score") == "sigmoid" or bias is not None or rule.get("groups", 1) > 1 else 28 * F32_STEP
    assert (np.abs(w.double().cpu().numpy() - rw) <= tol * np.abs(rw) + 2.0 ** -149).all()
    if plan:
        for got, want in zip((p.count, p.start, p.place), block.plan(ri, x.shape[1])):
            assert np.array_equal(got.cpu().numpy(), want)
    else:
        assert p is None
    return ids, w, p


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1, 1), (1, 8, 2), (3, 33, 32), (64, 128, 8), (65, 60, 4), (130, 512, 10), (1001, 8, 2), (700, 256, 8)])
def test_softmax_without_bias(tokens, experts, top_k, dtype):
    for renormalise in (True, False):
        check(logits_of(tokens, experts, dtype, tokens + experts), top_k, renormalise=renormalise, scale=1.0 if renormalise else 0.3)
    bd.poll_status()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("tokens,experts,top_k,groups,top_groups,group_top", [
    (5, 16, 4, 4, 2, 2), (64, 256, 8, 8, 4, 2), (100, 160, 6, 8, 3, 1), (257, 512, 10, 16, 5, 2), (70, 96, 3, 32, 1, 2), (70, 64, 8, 1, 1, 2), (33, 384, 8, 1, 1, 2), (9, 6, 2, 6, 2, 2)])
def test_bias_and_groups(tokens, experts, top_k, groups, top_groups, group_top, score):
    g = torch.Generator().manual_seed(experts)
    x = logits_of(tokens, experts, torch.float32, 3)
    for bias in (None, 0.1 * torch.randn(experts, generator=g)):
        for renormalise in (True, False):
            check(x, top_k, score=score, bias=bias, groups=groups, top_groups=top_groups, group_top=group_top, renormalise=renormalise, scale=2.5)
    bd.poll_status()


def test_equal_keys_go_to_the_lower_number():
    x = torch.zeros(70, 96)
    x[1::2] = torch.randint(0, 3, (35, 96), generator=torch.Generator().manual_seed(0)).float()
    x[5] = -0.0
    x[5, 40] = 0.0                                                # zeros of both signs are one number
    for rule in (dict(), dict(score="sigmoid"), dict(groups=8, top_groups=3), dict(score="sigmoid", groups=8, top_groups=3, group_top=1), dict(bias=torch.zeros(96))):
        check(x, 7, **rule)
    bd.poll_status()


def test_experts_that_are_not_there():
    x = logits_of(80, 40, torch.float32, 9)
    x[0] = -torch.inf                                             # a row without experts
    x[1, 3:] = -torch.inf                                         # fewer than are asked for
    x[2, ::2] = -torch.inf
    x[3, :10] = -torch.inf                                        # a whole group
    x[4, 1:10] = -torch.inf                                       # a group with one left
    x[5] = -1e30
    x[6] = torch.tensor([3e38, -3e38]).repeat(20)
    bias = torch.zeros(40)
    bias[7] = -torch.inf
    for rule in (dict(), dict(score="sigmoid"), dict(renormalise=False), dict(bias=bias), dict(bias=bias, score="sigmoid"), dict(groups=4, top_groups=2), dict(groups=4, top_groups=4, bias=bias, score="sigmoid", renormalise=False)):
        check(x, 5, **rule)
    bd.poll_status()


def test_what_is_not_a_number_is_told_and_never_chosen_before_numbers():
    for bad in (torch.nan, torch.inf):
        x = logits_of(66, 32, torch.float32, 1)
        x[3, 5] = bad
        x[65] = torch.nan
        for rule in (dict(), dict(bias=torch.zeros(32)), dict(score="sigmoid", groups=4, top_groups=2)):
            check(x, 4, **rule)
            with pytest.raises(bd.BdError) as e:
                bd.poll_status()
            assert e.value.status == 6
            bd.poll_status()
    b = torch.zeros(32)
    b[2] = torch.nan
    check(logits_of(4, 32, torch.float32, 1), 32, bias=b)
    with pytest.raises(bd.BdError):
        bd.poll_status()


@pytest.mark.parametrize("valid", [-3, 0, 1, 64, 65, 100, 200])
def test_padded_batches(valid):
    x = logits_of(100, 24, torch.float32, 4)
    x[max(0, min(valid, 100)):] = torch.nan                       # what stands behind the last token is not looked at
    check(x, 3, valid=valid)
    check(x[:50], 3, valid=valid)
    bd.poll_status()


def test_strided_logits_given_buffers_and_no_plan():
    x = logits_of(90, 64, torch.float32, 5)
    wide = torch.full((90, 101), torch.nan)
    wide[:, 20:84] = x
    dev = wide.cuda()[:, 20:84]
    want = bd.route(x.cuda(), 6)
    ids, w = torch.empty(90, 6, dtype=torch.int32, device="cuda"), torch.empty(90, 6, device="cuda")
    got = bd.route(dev, 6, ids=ids, weights=w, plan=want[2])
    assert got[0] is ids and got[1] is w and got[2] is want[2]
    assert torch.equal(ids, want[0]) and torch.equal(w, want[1])
    check(x, 6, plan=False)
    with pytest.raises(bd.BdError) as e:                          # rows that overlap
        bd.route(x.cuda()[:1].expand(70, 64), 6)
    assert e.value.status == 2


@pytest.mark.parametrize("tokens,experts,top_k", [(0, 4, 2), (1, 1, 1), (64, 7, 3), (65, 512, 1), (1000, 16, 4), (20000, 64, 2)])
def test_plans_of_given_ids(tokens, experts, top_k):
    ids = torch.randint(-2, experts, (tokens, top_k), generator=torch.Generator().manual_seed(tokens), dtype=torch.int32)
    if tokens > 3:
        ids[2] = ids[2, 0]                                        # a token that names an expert more than once
        ids[3] = -1
    if tokens > 10000:                                            # the oracle is slow: its sets by numpy
        ids[:, 1] = (ids[:, 0] + 1) % experts
    p = bd.expert_plan(ids.cuda(), experts)
    if tokens <= 1000:
        want = block.plan(ids.numpy(), experts)
    else:
        flat = ids.numpy()
        member = np.zeros((tokens, experts), bool)
        for j in range(top_k):
            ok = flat[:, j] >= 0
            member[np.nonzero(ok)[0], flat[ok, j]] = True
        count = member.sum(0)
        start = np.concatenate([[0], np.cumsum((count + 127) // 128 * 128)])
        rank = np.cumsum(member, 0) - member
        place = np.where(flat >= 0, start[np.maximum(flat, 0)] + np.take_along_axis(rank, np.maximum(flat, 0), 1), -1)
        want = count, start, place
    for got, w in zip((p.count, p.start, p.place), want):
        assert np.array_equal(got.cpu().numpy(), w)
    bd.poll_status()
    again = bd.expert_plan(ids.cuda(), experts, out=p)
    assert again is p


def test_ids_behind_the_last_expert_are_left_out_and_told():
    ids = torch.tensor([[0, 5], [4, 1], [2 ** 31 - 1, 3]], dtype=torch.int32)
    for reps in (1, 50):
        many = ids.repeat(reps, 1)
        p = bd.expert_plan(many.cuda(), 4)
        clean = torch.where(many < 4, many, -1)
        for got, want in zip((p.count, p.start, p.place), block.plan(clean.numpy(), 4)):
            assert np.array_equal(got.cpu().numpy(), want)
        with pytest.raises(bd.BdError) as e:
            bd.poll_status()
        assert e.value.status == 10


def test_captured_routing_follows_its_inputs():
    x = logits_of(150, 48, torch.float32, 6).cuda()
    valid = torch.tensor([150], dtype=torch.int32, device="cuda")
    bd.route(x, 4, valid=valid, score="sigmoid", groups=6, top_groups=2)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ids, w, p = bd.route(x, 4, valid=valid, score="sigmoid", groups=6, top_groups=2)
    for seed, n in ((7, 150), (8, 90), (9, 0)):
        fresh = logits_of(150, 48, torch.float32, seed)
        x.copy_(fresh)
        valid.fill_(n)
        g.replay()
        ri, rw = block.route(fresh.double().numpy(), 4, score="sigmoid", groups=6, top_groups=2, valid=n)
        assert np.array_equal(ids.cpu().numpy(), ri)
        for got, want in zip((p.count, p.start, p.place), block.plan(ri, 48)):
            assert np.array_equal(got.cpu().numpy(), want)


def test_many_tokens_and_another_stream():
    x = logits_of(70000, 64, torch.bfloat16, 11)                  # more blocks of 64 tokens than CTAs of the second launch
    s = torch.cuda.Stream()
    dev = x.cuda()
    s.wait_stream(torch.cuda.current_stream())
    ids, w, p = bd.route(dev, 3, stream=s)
    s.synchronize()
    order = torch.sort(x.double(), dim=-1, descending=True, stable=True)[1][:, :3]
    assert torch.equal(ids.cpu().long(), order)
    flat = order.reshape(-1)
    count = torch.bincount(flat, minlength=64)
    start = torch.cat([torch.zeros(1, dtype=torch.long), ((count + 127) // 128 * 128).cumsum(0)])
    by = torch.sort(flat, stable=True)[1]
    place = torch.empty_like(flat)
    place[by] = start[flat[by]] + torch.arange(len(flat)) - (count.cumsum(0) - count)[flat[by]]
    assert torch.equal(p.count.cpu().long(), count) and torch.equal(p.start.cpu().long(), start) and torch.equal(p.place.cpu().long().reshape(-1), place)
