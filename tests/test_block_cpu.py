"""Routing, experts and norms without a GPU: refusals of the C entry points and of the binding, sizes, and the oracle's pins."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from oracle import block
from paper_2501_01144_b200 import binding

vp, i64 = ctypes.c_void_p, ctypes.c_int64


class Rule(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int), ("experts", i64), ("top_k", i64), ("groups", i64), ("top_groups", i64), ("group_top", ctypes.c_int), ("renormalise", ctypes.c_int), ("scale", ctypes.c_float)]


class Plan(ctypes.Structure):
    _fields_ = [("count", vp), ("start", vp), ("place", vp), ("scratch", vp), ("tokens", i64), ("top_k", i64), ("experts", i64)]


class Experts(ctypes.Structure):
    _fields_ = [("codes", vp), ("ids", vp), ("scales", vp), ("experts", i64), ("rows", i64), ("K", i64)]


class Norm(ctypes.Structure):
    _fields_ = [(n, vp) for n in ("y", "residual", "gate", "post_weight", "post_bias", "weight", "bias")] + [(n, i64) for n in ("ldy", "ld_residual", "gate_row", "gate_col")] + \
        [(n, ctypes.c_float) for n in ("scale", "eps", "weight_offset")] + [("layer", ctypes.c_int), ("h", vp), ("n", vp), ("ldh", i64), ("ldn", i64), ("q", vp)]


def lib():
    lib = bd.load()
    lib.bd_route.argtypes = [vp, ctypes.c_int, i64, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.bd_make_expert_plan.argtypes = [vp, vp, vp]
    lib.bd_expert_plan_scratch.argtypes = [i64, i64, vp]
    lib.bd_expert_mlp_workspace_size.argtypes = [i64, i64, vp, vp, ctypes.c_int, vp]
    lib.bd_expert_mlp.argtypes = [vp, ctypes.c_int, i64, i64, vp, vp, vp, vp, ctypes.c_int, vp, ctypes.c_int, i64, vp, vp, ctypes.c_size_t, vp]
    lib.bd_residual_norm.argtypes = [vp, ctypes.c_int, i64, i64, vp]
    return lib


@pytest.mark.parametrize("change,status", [
    (dict(score=2), 1), (dict(experts=0), 1), (dict(top_k=0), 1), (dict(groups=0), 1), (dict(top_groups=0), 1), (dict(group_top=0), 1), (dict(group_top=3), 1), (dict(scale=float("inf")), 1),
    (dict(scale=float("nan")), 1), (dict(top_k=65), 2), (dict(groups=5), 2), (dict(groups=4, top_groups=5), 2), (dict(ld=63), 2), (dict(experts=1024, ld=1024), 4), (dict(top_k=33), 4), (dict(groups=64), 4),
    (dict(tokens=-1), 1), (dict(tokens=2 ** 31), 4), (dict(dtype=3), 1), (dict(logits=0), 1), (dict(ids=0), 1), (dict(weights=0), 1), (dict(logits=0x1002), 3), (dict(bias=0x1002), 3), (dict(ids=0x1001), 3),
    (dict(plan_tokens=99), 2), (dict(plan_k=5), 2), (dict(plan_experts=32), 2), (dict(scratch=0), 8), (dict(scratch=0x1008), 3), (dict(place=0), 1), (dict(count=0x1001), 3)])
def test_route_refuses_before_any_launch(change, status):
    a = dict(score=0, experts=64, top_k=4, groups=1, top_groups=1, group_top=2, scale=1.0, ld=64, tokens=100, dtype=0, logits=0x1000, bias=0x1000, ids=0x1000, weights=0x1000, plan_tokens=None, plan_k=None,
             plan_experts=None, scratch=0x1000, place=0x1000, count=0x1000)
    a.update(change)
    rule = Rule(a["score"], a["experts"], a["top_k"], a["groups"], a["top_groups"], a["group_top"], 1, a["scale"])
    plan = Plan(a["count"], 0x1000, a["place"], a["scratch"], a["tokens"] if a["plan_tokens"] is None else a["plan_tokens"], a["plan_k"] or a["top_k"], a["plan_experts"] or a["experts"])
    assert lib().bd_route(a["logits"], a["dtype"], a["tokens"], a["ld"], a["bias"], ctypes.byref(rule), None, a["ids"], a["weights"], ctypes.byref(plan), None) == status
    assert lib().bd_route(0x1000, 0, 1, 64, None, None, None, 0x1000, 0x1000, None, None) == 1


def test_plan_refusals_and_scratch():
    n = ctypes.c_size_t()
    assert lib().bd_expert_plan_scratch(64, 60, ctypes.byref(n)) == 0 and n.value == 0
    assert lib().bd_expert_plan_scratch(65, 60, ctypes.byref(n)) == 0 and n.value == 2 * 64
    assert lib().bd_expert_plan_scratch(8192, 256, ctypes.byref(n)) == 0 and n.value == 128 * 256
    assert lib().bd_expert_plan_scratch(-1, 4, ctypes.byref(n)) == 1 and lib().bd_expert_plan_scratch(1, 0, ctypes.byref(n)) == 1 and lib().bd_expert_plan_scratch(1, 513, ctypes.byref(n)) == 4
    make = lambda ids, **k: lib().bd_make_expert_plan(ids, ctypes.byref(Plan(*[{**dict(count=0x1000, start=0x1000, place=0x1000, scratch=0x1000, tokens=100, top_k=2, experts=8), **k}[f] for f, _ in Plan._fields_])), None)  # noqa: E731
    assert make(0) == 1 and make(0x1001) == 3 and make(0x1000, count=0) == 1 and make(0x1000, experts=0) == 1 and make(0x1000, experts=513) == 4 and make(0x1000, top_k=33) == 4
    assert make(0x1000, tokens=2 ** 30) == 4 and make(0x1000, scratch=0) == 8 and make(0x1000, scratch=0x1004) == 3 and make(0x1000, start=0x1002) == 3


def expert_args(**change):
    a = dict(tokens=100, k=2, experts=8, hidden=256, inter=128, n=264, up_rows=None, down_experts=None, x=0x1000, xdtype=1, ldx=256, weights=0x1000, act=0, y=0x1000, ydtype=1, ldy=264, inner=None, ws=0x1000,
             ws_bytes=1 << 40, plan_tokens=None, plan_experts=None, codes=0x1000)
    a.update(change)
    up = Experts(a["codes"], 0x1000, 0x1000, a["experts"], 2 * a["inter"] if a["up_rows"] is None else a["up_rows"], a["hidden"])
    down = Experts(0x1000, 0x1000, 0x1000, a["down_experts"] or a["experts"], a["n"], a["inter"])
    plan = Plan(0x1000, 0x1000, 0x1000, 0x1000, a["tokens"] if a["plan_tokens"] is None else a["plan_tokens"], a["k"], a["plan_experts"] or a["experts"])
    return a, up, down, plan


@pytest.mark.parametrize("change,status", [
    (dict(hidden=250, ldx=256), 2), (dict(inter=120), 2), (dict(n=260), 2), (dict(up_rows=128), 2), (dict(down_experts=7), 2), (dict(experts=513), 4), (dict(codes=0), 1), (dict(codes=0x1008), 3), (dict(x=0), 1),
    (dict(y=0), 1), (dict(weights=0), 1), (dict(x=0x1008), 3), (dict(y=0x1008), 3), (dict(ldx=255), 2), (dict(ldx=260), 3), (dict(ldy=260), 2), (dict(ldy=270), 3), (dict(xdtype=5), 1), (dict(ydtype=2), 1),
    (dict(act=2), 1), (dict(plan_tokens=99), 2), (dict(plan_experts=9), 2), (dict(ws=0), 8), (dict(ws_bytes=1000), 8), (dict(ws=0x1010), 3), (dict(inner=0x1002), 3), (dict(k=33), 4), (dict(weights=0x1002), 3),
    (dict(tokens=2 ** 29, plan_tokens=2 ** 29, k=2), 4)])
def test_expert_mlp_refuses_before_any_launch(change, status):
    a, up, down, plan = expert_args(**change)
    assert lib().bd_expert_mlp(a["x"], a["xdtype"], a["tokens"], a["ldx"], ctypes.byref(plan), a["weights"], ctypes.byref(up), ctypes.byref(down), a["act"], a["y"], a["ydtype"], a["ldy"], a["inner"], a["ws"],
                               a["ws_bytes"], None) == status


def test_expert_workspace_follows_its_parts():
    n = ctypes.c_size_t()

    def size(ydtype=1, **change):
        a, up, down, _ = expert_args(**change)
        assert lib().bd_expert_mlp_workspace_size(a["tokens"], a["k"], ctypes.byref(up), ctypes.byref(down), ydtype, ctypes.byref(n)) == 0
        return n.value

    up256 = lambda x: (x + 255) // 256 * 256  # noqa: E731
    rows = (200 + 127 * 8) // 128 * 128                           # each expert's rows rounded up to 128, at worst
    scales = lambda k: rows // 128 * -(-k // 128) * 512  # noqa: E731
    assert size() == up256(rows * 264 * 2) + scales(256) + up256(rows * 128) + scales(128)
    assert size(ydtype=0) == up256(rows * 264 * 4) + scales(256) + up256(rows * 128) + scales(128)
    assert size(n=8) == up256(rows * 256) + scales(256) + up256(rows * 128) + scales(128)
    assert size(tokens=0) == 0
    rows = 128                                                    # one token, one expert
    assert size(tokens=1, k=1) == up256(rows * 264 * 2) + scales(256) + up256(rows * 128) + scales(128)


@pytest.mark.parametrize("change,status", [
    (dict(y=0), 1), (dict(h=0, n=0), 1), (dict(weight=0), 1), (dict(post_weight=0, post_bias=0x1000), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(weight_offset=float("nan")), 1), (dict(gate=0x1000, gate_col=2), 1), (dict(gate=0x1000, gate_row=-1), 1), (dict(h=0x1000, n=0x1000), 1), (dict(ldy=63), 2), (dict(residual=0x1000, ld_residual=1), 2),
    (dict(ldh=10), 2), (dict(ldn=10), 2), (dict(y=0x1002), 3), (dict(weight=0x1001), 3), (dict(gate=0x1002), 3), (dict(dim=16385, ldy=20000, ldh=20000, ldn=20000), 4), (dict(dim=0), 1), (dict(rows=-1), 1),
    (dict(rows=2 ** 31), 4), (dict(dtype=7), 1)])
def test_residual_norm_refuses_before_any_launch(change, status):
    a = dict(y=0x1000, weight=0x1000, h=0x1000, n=0x2000, ldy=64, ldh=64, ldn=64, eps=1e-6, scale=1.0, rows=4, dim=64, dtype=0)
    a.update(change)
    s = Norm(**{k: v for k, v in a.items() if k not in ("rows", "dim", "dtype")})
    assert lib().bd_residual_norm(ctypes.byref(s), a["dtype"], a["rows"], a["dim"], None) == status


def test_residual_norm_checks_the_operand_it_quantises_into():
    q = binding._CQTensor(0x1000, 0x1000, 0x1000, 4, 64)
    call = lambda dim, rows, qt, n=0: lib().bd_residual_norm(ctypes.byref(Norm(y=0x1000, weight=0x1000, ldy=512, n=n, ldn=512, q=ctypes.addressof(qt))), 0, rows, dim, None)  # noqa: E731
    assert call(64, 5, q) == 2 and call(96, 4, q) == 2 and call(64, 4, q, 0x2000) == 1
    assert call(64, 4, binding._CQTensor(0x1000, 0x1000, 0x1008, 4, 64)) == 3 and call(40, 4, binding._CQTensor(0x1000, 0x1000, 0x1000, 4, 40)) == 2


def test_the_binding_refuses_what_it_is_not_given_right():
    x = torch.zeros(4, 8)
    for call in (lambda: bd.route(x, 2, score="other"), lambda: bd.route(x, 9), lambda: bd.route(x, 0), lambda: bd.route(x[0], 1), lambda: bd.route(x.long(), 1), lambda: bd.route(None, 1),
                 lambda: bd.expert_plan(torch.zeros(4, 2), 4), lambda: bd.expert_plan(torch.zeros(4, dtype=torch.int32), 4), lambda: bd.residual_norm(x, None, norm="other"),
                 lambda: bd.residual_norm(x[0], None), lambda: bd.residual_norm(x[0], None, quantise=True), lambda: bd.residual_norm(x.long(), None), lambda: bd.quantize_experts(x), lambda: bd.quantize_experts(torch.zeros(1, 96, 32), gated=True)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises((ValueError, RuntimeError)):               # a tensor that is not on the GPU
        bd.route(x, 2)


def test_oracle_routes_as_by_hand():
    x = np.array([[1.0, 3.0, 2.0, 3.0], [0.0, -np.inf, -np.inf, -np.inf], [-np.inf] * 4])
    ids, w = block.route(x, 2)
    assert ids.tolist() == [[1, 3], [0, -1], [-1, -1]] and np.allclose(w, [[0.5, 0.5], [1, 0], [0, 0]])
    ids, w = block.route(x[:1], 2, bias=np.array([5.0, 0, 0, 0]), renormalise=False)
    p = np.exp(x[0] - 3) / np.exp(x[0] - 3).sum()
    assert ids.tolist() == [[0, 1]] and np.allclose(w, p[[0, 1]])
    # groups {0, 1}, {2, 3}: the sum of two decides for the second, the largest one for the first
    y = np.array([[3.0, -9.0, 2.5, 2.4]])
    assert block.route(y, 1, score="sigmoid", groups=2, top_groups=1)[0].tolist() == [[2]] and block.route(y, 1, score="sigmoid", groups=2, top_groups=1, group_top=1)[0].tolist() == [[0]]


def test_oracle_plan_as_by_hand():
    count, start, place = block.plan(np.array([[1, 0], [1, -1], [1, 1]]), 3)
    assert count.tolist() == [1, 3, 0] and start.tolist() == [0, 128, 256, 256] and place.tolist() == [[128, 0], [129, -1], [130, 130]]
    assert block.gated_order(64)[[0, 31, 32, 63, 64, 96]].tolist() == [0, 31, 64, 95, 32, 96]


def test_plain_forms_of_the_cases_agree_with_the_oracle():
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf"))
    import more_operators as m
    x = torch.randn(50, 24, generator=torch.Generator().manual_seed(0))
    bias = 0.1 * torch.randn(24, generator=torch.Generator().manual_seed(1))
    case = dict(op="route", experts=24, top_k=3, score="sigmoid", groups=4, top_groups=2, renormalise=True, scale=1.5)
    ids, w, count, place = m.run(dict(case=case, logits=x, bias=bias))
    ri, rw = block.route(x.double().numpy(), 3, score="sigmoid", bias=bias.double().numpy(), groups=4, top_groups=2, scale=1.5)
    assert np.array_equal(ids.numpy(), ri) and np.abs(w.numpy() - rw).max() < 1e-6
    rc, _, rp = block.plan(ri, 24)
    assert np.array_equal(count.numpy(), rc) and np.array_equal(place.numpy(), rp)
