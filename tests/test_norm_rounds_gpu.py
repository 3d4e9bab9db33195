"""The norms where a CTA goes through many rows: the last row numbers, further rounds of rows, and quantised rows of every kind."""
import pytest
import torch

import paper_2501_01144_b200 as bd

pytestmark = pytest.mark.gpu


def test_as_many_rows_as_there_can_be():
    rows, guard = 2 ** 31 - 1 - 128, 1 << 20
    y = torch.empty(rows + guard, dtype=torch.float16, device="cuda")
    for at in range(0, rows + guard, 1 << 28):
        part = y[at:at + (1 << 28)]
        part.copy_((torch.arange(at, at + part.numel(), device="cuda") % 1999).half())
    h = torch.full_like(y, 7.0)
    bd.residual_norm(y[guard:, None], None, scale=0.5, out_h=h[guard:, None])
    assert (h[:guard] == 7).all()
    for at in range(guard, rows + guard, 1 << 28):
        assert torch.equal(h[at:at + (1 << 28)], y[at:at + (1 << 28)] * 0.5)
    bd.poll_status()


STEP = 2.0 ** -24                                                 # half a step of fp32, relative


def normed(x, ex, w, layer, eps):
    """(norm in 64 bits, bound of the fp32 error) of x known within ex: a row's sum is at most 32 additions in a thread and 10 levels across
    threads, of terms of one sign (42 half steps); the root halves the sum's error and adds 2 steps; then three products."""
    if layer:
        ex = ex + 44 * STEP * x.abs().mean(-1, keepdim=True) + STEP * x.abs()
        x = x - x.mean(-1, keepdim=True)
    f = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    y = x * f * w
    return y, f * w.abs() * ex + y.abs() * (f * ex.square().mean(-1, keepdim=True).sqrt() + 30 * STEP)


# a CTA has 2048 threads' worth of rows at a time: pieces of eight elements, one, two and four a thread, rows that share a CTA, rows of odd length
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("rows,dim,dtype", [(20000, 96, torch.float32), (30000, 512, torch.bfloat16), (7000, 768, torch.float16), (7000, 515, torch.bfloat16), (6000, 4096, torch.bfloat16), (2000, 2559, torch.float32),
                                            (1500, 8192, torch.float32), (1300, 16384, torch.bfloat16), (25000, 7, torch.float16)])
def test_several_rounds_of_rows(rows, dim, dtype, layer):
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    y, residual, gate = r(rows, dim).to(dtype), (3 * r(rows, dim)).to(dtype), torch.sigmoid(r(rows, 1)).to(dtype)
    w, post = (1 + 0.2 * r(dim)).to(dtype), (1 + 0.2 * r(dim)).to(dtype)
    kw = dict(post_weight=post, gate=gate, norm="layer" if layer else "rms", eps=1e-5)
    h, n = bd.residual_norm(y, w, residual, **kw)
    half, tiny = torch.finfo(dtype).eps / 2, {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -126}[dtype]
    for at in range(0, rows, 4096):
        part = slice(at, at + 4096)
        u, e = normed(y[part].double(), torch.zeros((), dtype=torch.float64, device="cuda").expand(len(y[part]), dim), post.double(), layer, 1e-5)
        u, e = gate[part].double() * u, gate[part].double() * e
        want = u + residual[part].double()
        e = e + 3 * STEP * u.abs() + STEP * want.abs() + 2.0 ** -126
        assert ((h[part].double() - want).abs() <= e + half * (want.abs() + e) + tiny).all()
        want, e = normed(want, e, w.double(), layer, 1e-5)
        assert ((n[part].double() - want).abs() <= e + half * (want.abs() + e) + tiny).all()
    # in place, and with strided rows: the next rows are on their way while these are written
    wide = torch.full((rows, dim + 8), 5.0, dtype=dtype, device="cuda")
    wide[:, :dim] = y
    res = residual.clone()
    bd.residual_norm(wide[:, :dim], w, res, out_h=res, out_n=wide[:, :dim], **kw)
    if dtype == torch.float32 or dim % 8 == 0:                    # (rows of the same alignment: the same order of sums)
        assert torch.equal(res, h) and torch.equal(wide[:, :dim], n)
    assert (wide[:, dim:] == 5).all()
    y2, res2 = y.clone(), residual.clone()
    bd.residual_norm(y2, w, res2, out_h=y2, out_n=res2, **kw)
    assert torch.equal(y2, h) and torch.equal(res2, n)
    bd.poll_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,dim", [(296, 128), (297, 32), (300, 1024), (700, 96), (2000, 4096), (20000, 160), (20000, 1024), (1500, 8192), (700, 16384)])
def test_quantised_rows_of_every_number(rows, dim, dtype):
    # whole numbers whose squares add up exactly in fp32: the sums have no order, so the normalised rows that are quantised are those that are stored
    g = torch.Generator(device="cuda").manual_seed(rows)
    i = lambda: torch.randint(-4, 5, (rows, dim), generator=g, device="cuda").to(dtype)  # noqa: E731
    y, residual, w = i(), i(), (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dtype)
    h, n = bd.residual_norm(y, w, residual)
    out = bd.QTensor(rows, dim)
    want = bd.QTensor(rows, dim)
    for q in (out, want):
        for b in (q.codes, q.ids, q.scales):
            b.fill_(0xff)
    bd.quantize_act(n, out=want)

    def same(q):
        return torch.equal(q.codes, want.codes) and torch.equal(q.ids, want.ids) and torch.equal(q.scales, want.scales)

    h2, q = bd.residual_norm(y, w, residual, quantise=True, out_n=out)
    assert q is out and torch.equal(h2, h) and same(out)
    res = residual.clone()
    assert same(bd.residual_norm(y, w, res, quantise=True, out_h=res, out_n=out)[1]) and torch.equal(res, h)
    wide = torch.full((rows, dim + 3), float("nan"), dtype=dtype, device="cuda")   # rows off a 16-byte boundary: single elements
    wide[:, 3:] = y
    assert same(bd.residual_norm(wide[:, 3:], w, residual, quantise=True, want_h=False)[1])
    bd.poll_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,dim", [(1, 32), (5, 416), (130, 128), (700, 96), (2500, 1024), (3, 16384)])
def test_quantised_rows_off_a_boundary_have_the_bits_of_storing_and_quantising(rows, dim, dtype):
    # any numbers: the stored and the quantised result of such rows come from the same sums in the same order
    g = torch.Generator(device="cuda").manual_seed(rows + dim)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    y, residual, w, post, gate = r(rows, dim + 1)[:, 1:], r(rows, dim), r(dim), r(dim), r(rows, dim)
    for norm in ("rms", "layer"):
        h, n = bd.residual_norm(y, w, residual, post_weight=post, gate=gate, norm=norm)
        h2, q = bd.residual_norm(y, w, residual, post_weight=post, gate=gate, norm=norm, quantise=True)
        want = bd.quantize_act(n)
        assert torch.equal(h, h2) and torch.equal(q.codes, want.codes) and torch.equal(q.ids, want.ids) and torch.equal(q.scales, want.scales)
    bd.poll_status()


def test_a_quantised_result_needs_a_row():
    w = torch.ones(64, device="cuda")
    with pytest.raises(bd.BdError) as e:
        bd.residual_norm(torch.empty(0, 64, device="cuda"), w, quantise=True)
    assert e.value.status == 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,dim", [(297, 4096), (700, 96), (2000, 4096), (1000, 1024), (1000, 2080), (20000, 512), (3000, 8192), (1000, 16384)])
def test_stored_and_quantised_rows_have_the_same_sums(rows, dim, dtype):
    # any numbers, two norms: the quantised result is that of the stored one, and a row's does not depend on the other rows
    g = torch.Generator(device="cuda").manual_seed(rows + dim)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    y, residual, w, post, gate, bias = r(rows, dim), r(rows, dim), r(dim), r(dim), r(rows, dim), r(dim)
    for kw in (dict(post_weight=post, gate=gate), dict(post_weight=post, post_bias=bias, bias=bias, norm="layer", weight_offset=1.0)):
        h, n = bd.residual_norm(y, w, residual, **kw)
        h2, q = bd.residual_norm(y, w, residual, quantise=True, **kw)
        want = bd.quantize_act(n)
        assert torch.equal(h, h2) and torch.equal(q.codes, want.codes) and torch.equal(q.ids, want.ids) and torch.equal(q.scales, want.scales)
        for at, to in ((0, 1), (rows // 2, rows // 2 + 3), (rows - 296, rows)):
            some = {**kw, **({"gate": gate[at:to]} if "gate" in kw else {})}
            h3, n3 = bd.residual_norm(y[at:to], w, residual[at:to], **some)
            assert torch.equal(h3, h[at:to]) and torch.equal(n3, n[at:to])
    bd.poll_status()
