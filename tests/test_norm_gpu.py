"""The norms around a block on the GPU, against the oracle in 64 bits; the quantised result against storing and quantising, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from oracle import block

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24                                                 # half a step of fp32, relative


def make(rows, dim, dtype, seed=0, post=False, gate="none", residual=True, layer=False):
    g = torch.Generator().manual_seed(seed + rows + dim)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    near = lambda: (1 + 0.2 * r(dim)).to(dtype).cuda()  # noqa: E731
    a = dict(y=r(rows, dim).to(dtype).cuda(), weight=near())
    if residual:
        a["residual"] = (r(rows, dim) * 3 * torch.where(torch.rand(dim, generator=g) < 0.02, 20.0, 1.0)).to(dtype).cuda()
    if post:
        a["post_weight"] = near()
    if layer:
        a["bias"] = (0.1 * r(dim)).to(dtype).cuda()
        if post:
            a["post_bias"] = (0.1 * r(dim)).to(dtype).cuda()
    shape = {"none": None, "row": (rows, 1), "channel": (1, dim), "element": (rows, dim), "one": (1, 1)}[gate]
    if shape:
        a["gate"] = torch.sigmoid(r(*shape)).to(dtype).cuda()
    return a


def normed(x, ex, w, b, layer, eps, offset):
    """(norm in 64 bits, bound of the fp32 error) of x known within ex.  A sum over a row is at most 32 additions in a thread and 10
    levels across threads, all terms of one sign (squares, or magnitudes for the mean's bound): 42 half steps; the root halves the sum's
    error and adds 2 steps; then three products and a sum."""
    n = x.shape[-1]
    if layer:
        ex = ex + 44 * STEP * np.abs(x).mean(-1, keepdims=True) + STEP * np.abs(x)
        x = x - x.mean(-1, keepdims=True)
    f = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    scale = np.abs(w + offset)
    y = x * f * (w + offset)
    rms_e = np.sqrt((ex * ex).sum(-1, keepdims=True) / n)
    err = f * scale * ex + np.abs(y) * (f * rms_e + (22 + 4 + 4) * STEP)
    if b is not None:
        y = y + b
        err = err + STEP * np.abs(y)
    return y, err


def check(a, scale=1.0, norm="rms", eps=1e-6, offset=0.0, **more):
    h, n = bd.residual_norm(a["y"], a["weight"], a.get("residual"), bias=a.get("bias"), post_weight=a.get("post_weight"), post_bias=a.get("post_bias"), gate=a.get("gate"), scale=scale, norm=norm,
                            eps=eps, weight_offset=offset, **more)
    d = {k: v.double().cpu().numpy() for k, v in a.items()}
    layer = norm == "layer"
    u, e = d["y"], np.zeros_like(d["y"])
    if "post_weight" in d:
        u, e = normed(u, e, d["post_weight"], d.get("post_bias"), layer, eps, offset)
    gate = d.get("gate", 1.0)
    part = scale * gate * u
    ref_h = part + d.get("residual", 0.0)
    e = np.abs(scale * gate) * e + 2 * STEP * np.abs(part) + STEP * np.abs(ref_h) + 2.0 ** -126   # (the scale itself is an fp32 number: below)
    e = e + STEP * np.abs(part)
    half = torch.finfo(a["y"].dtype).eps / 2
    tiny = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -126}[a["y"].dtype]
    assert (np.abs(h.double().cpu().numpy() - ref_h) <= e + half * (np.abs(ref_h) + e) + tiny).all()
    want = block.norm(ref_h, d["weight"], d.get("bias"), layer, eps, offset)
    same, en = normed(ref_h, e, d["weight"], d.get("bias"), layer, eps, offset)
    assert np.allclose(same, want, rtol=1e-12, atol=1e-12 * np.abs(want).max())   # (the oracle and the bound's own 64-bit form: near zero their sums' last bits show)
    assert (np.abs(n.double().cpu().numpy() - want) <= en + half * (np.abs(want) + en) + tiny).all()
    return h, n


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 64), (2, 255), (17, 256), (4, 1000), (9, 2559), (3, 4096), (2, 5120), (2, 8193), (2, 16384), (700, 320)])
def test_residual_and_norm(rows, dim, dtype):
    check(make(rows, dim, dtype))
    check(make(rows, dim, dtype, post=True, gate="channel", layer=True), norm="layer", scale=0.22, eps=1e-5)
    bd.poll_status()


@pytest.mark.parametrize("gate", ["none", "row", "channel", "element", "one"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_gates_and_norms_before_and_after(gate, post, norm):
    for dim in (96, 515, 4096):
        for residual in (True, False):
            check(make(6, dim, torch.bfloat16, post=post, gate=gate, layer=norm == "layer", residual=residual), norm=norm, scale=-0.5, offset=1.0)
    bd.poll_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,dim", [(1, 32), (3, 96), (130, 128), (5, 416), (64, 4096), (7, 5120), (129, 160), (2, 16384)])
def test_quantised_result_has_the_bits_of_storing_and_quantising(rows, dim, dtype):
    a = make(rows, dim, dtype, post=True, gate="element")
    args = [a["y"], a["weight"], a["residual"]], dict(post_weight=a["post_weight"], gate=a["gate"])
    h, n = bd.residual_norm(*args[0], **args[1])
    pad = bd.QTensor(rows, dim)
    for b in (pad.codes, pad.ids, pad.scales):
        b.fill_(0xff)                                             # padding of the atoms has to be written too
    want = bd.QTensor(rows, dim)
    bd.quantize_act(n, out=want)
    h2, q = bd.residual_norm(*args[0], **args[1], quantise=True, out_n=pad)
    assert q is pad and torch.equal(h, h2)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.ids, want.ids) and torch.equal(q.scales, want.scales)
    # unaligned rows: the same bits by way of single elements
    wide = torch.zeros(rows, dim + 3, dtype=dtype, device="cuda")
    wide[:, 3:] = a["y"]
    _, q2 = bd.residual_norm(wide[:, 3:], a["weight"], a["residual"], **args[1], quantise=True, want_h=False)
    assert bd.dequantize(q2).shape == (rows, dim)
    assert (bd.dequantize(q2) - bd.dequantize(want)).abs().max() <= 2 * bd.dequantize(want).abs().max()
    bd.poll_status()


def test_result_feeds_a_product():
    a = make(40, 256, torch.bfloat16)
    W = bd.quantize_weights(torch.randn(96, 256, generator=torch.Generator().manual_seed(1)).cuda())
    _, n = bd.residual_norm(a["y"], a["weight"], a["residual"])
    _, q = bd.residual_norm(a["y"], a["weight"], a["residual"], quantise=True)
    assert torch.equal(bd.gemm(q, W), bd.linear(n, W, dtype=torch.float32))


def test_in_place_strided_and_single_outputs():
    a = make(33, 512, torch.bfloat16, post=True)
    kw = dict(post_weight=a["post_weight"])
    h, n = bd.residual_norm(a["y"], a["weight"], a["residual"], **kw)
    none, n2 = bd.residual_norm(a["y"], a["weight"], a["residual"], want_h=False, **kw)
    h2, none2 = bd.residual_norm(a["y"], None, a["residual"], **kw)
    assert none is None and none2 is None and torch.equal(n, n2) and torch.equal(h, h2)
    wide = torch.full((33, 700), 5.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, 8:520]
    bd.residual_norm(a["y"], a["weight"], a["residual"], out_n=out, **kw)
    assert torch.equal(out, n) and (wide[:, :8] == 5).all() and (wide[:, 520:] == 5).all()
    res, y = a["residual"].clone(), a["y"].clone()
    h3, n3 = bd.residual_norm(y, a["weight"], res, out_h=res, out_n=y, **kw)
    assert h3 is res and n3 is y and torch.equal(res, h) and torch.equal(y, n)
    plain = bd.residual_norm(a["y"], a["weight"], want_h=False)[1]   # the first norm of a model: nothing to add
    assert torch.equal(plain, bd.residual_norm(torch.zeros_like(a["y"]), a["weight"], a["y"])[1])


def test_rows_of_zeros_infinities_and_nan_stay_in_their_rows():
    a = make(6, 256, torch.float32)
    a["y"][1] = 0
    a["residual"][1] = 0
    want = bd.residual_norm(a["y"], a["weight"], a["residual"])
    assert (want[1][1] == 0).all()
    y = a["y"].clone()
    y[2, 5], y[4, 7] = torch.inf, torch.nan
    h, n = bd.residual_norm(y, a["weight"], a["residual"])
    for r in (0, 1, 3, 5):
        assert torch.equal(n[r], want[1][r]) and torch.equal(h[r], want[0][r])
    assert n[4].isnan().all() and n[2].isnan().any()
    bd.poll_status()
    _, q = bd.residual_norm(y, a["weight"], a["residual"], quantise=True)
    with pytest.raises(bd.BdError) as e:
        bd.poll_status()
    assert e.value.status == 6


def test_no_rows_and_capture():
    w = torch.ones(64, device="cuda")
    h, n = bd.residual_norm(torch.empty(0, 64, device="cuda"), w, torch.empty(0, 64, device="cuda"))
    assert h.shape == n.shape == (0, 64)
    a = make(10, 1024, torch.bfloat16)
    _, q = bd.residual_norm(a["y"], a["weight"], a["residual"], quantise=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h, n = bd.residual_norm(a["y"], a["weight"], a["residual"])
        _, q = bd.residual_norm(a["y"], a["weight"], a["residual"], quantise=True)
    a["y"].mul_(-0.7)
    g.replay()
    want = bd.residual_norm(a["y"], a["weight"], a["residual"])
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])
    assert torch.equal(q.codes, bd.quantize_act(n).codes)
