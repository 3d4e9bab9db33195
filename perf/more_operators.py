"""The operators of a mixture-of-experts block in DialectFP4, their plain forms and the cases they are timed on.

  route    a step's router logits: each token's experts, their weights, and where its rows lie among the experts' rows;
  experts  the chosen experts' gated products, weighted and added up;
  norm     the residual sum behind a block (its result normalised, gated and scaled on request) and the next block's norm,
           whose result may be a DialectFP4 operand.

`run` computes an operator from what `prepare` made: in plain torch operations, or (own = True) by the library's calls.

Storage of the experts' weights.  Expert after expert, each an operand [rows, K] of its own.  Codes [rows][K / 2] bytes: of each 8
elements byte b holds the indices of elements 2 b (bits 0 .. 2) and 2 b + 1 (bits 4 .. 6), the sign of element 4 + b (bit 3) and that
of element b (bit 7).  Scales (e + 127): atoms of 128 rows x 4 blocks of 32, atom (b / 4) * tiles + r / 128; in an atom (row r, block b)
is byte (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4.  Ids in atoms of the same order: nibble b % 2 of byte (r % 32) * 8 +
(r % 128 / 32) * 2 + b % 4 / 2.  Padding of atoms holds zeros.  The first product's rows alternate in groups of 32: rows 64 j .. 64 j + 31
are gate rows 32 j .. 32 j + 31, the next 32 the up rows of the same numbers.

Places.  Expert e has rows start[e] .. start[e] + count[e] - 1, in the order of its tokens; starts are multiples of 128.  An
assignment without an expert has place -1.
"""
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# The DialectFP4 formatbook in units of 0.5: pair p has the maximum 15 - p, and its members differ in their second largest value.
_SECOND = ((12, 10), (11, 9), (10, 8), (9, 8), (9, 8), (8, 7), (8, 7), (7, 6))
BOOK = [[0, 1, 2, 3, 4, 5 if p == 7 else 6, _SECOND[p][o], 15 - p] for p in range(8) for o in range(2)]


# ---- the cases ------------------------------------------------------------------------------------------------------


def listed():
    return [
        # one decode step of 64 sequences: latency
        dict(name="route 64 of 128", op="route", tokens=64, experts=128, top_k=8, score="softmax", bias=False, groups=1, top_groups=1, renormalise=True, scale=1.0, dtype="f32"),
        # a prefill batch, experts in groups, a bias that balances their load
        dict(name="route 8192 of 256 grouped", op="route", tokens=8192, experts=256, top_k=8, score="sigmoid", bias=True, groups=8, top_groups=4, renormalise=True, scale=2.5, dtype="f32"),
        # an odd batch over a few large experts, logits in 16 bits
        dict(name="route 1001 of 8 bf16", op="route", tokens=1001, experts=8, top_k=2, score="softmax", bias=False, groups=1, top_groups=1, renormalise=False, scale=1.0, dtype="bf16"),
        # one token: latency
        dict(name="experts 1 of 64", op="experts", tokens=1, experts=64, top_k=8, hidden=2048, inter=1024, act="silu", dtype="bf16", skew=0.5),
        # a decode step of 64 sequences over many small experts
        dict(name="experts 64 of 128", op="experts", tokens=64, experts=128, top_k=8, hidden=2048, inter=1024, act="silu", dtype="bf16", skew=0.5),
        # a ragged batch of middle size, sizes that are no multiples of a tile, fp16
        dict(name="experts 1500 of 64 f16", op="experts", tokens=1500, experts=64, top_k=6, hidden=2048, inter=1408, act="gelu", dtype="f16", skew=1.0),
        # a prefill batch over a few large experts
        dict(name="experts 8192 of 8", op="experts", tokens=8192, experts=8, top_k=2, hidden=4096, inter=14336, act="silu", dtype="bf16", skew=0.3),
        # one decode step: residual sum and the next block's operand in 4 bits
        dict(name="norm 64 rows quantised", op="norm", rows=64, dim=4096, kind="rms", post=False, gate="none", scale=1.0, quantise=True, offset=0.0, dtype="bf16"),
        # a prefill batch, norms before and after the block
        dict(name="norm 8192 rows", op="norm", rows=8192, dim=4096, kind="rms", post=True, gate="none", scale=1.0, quantise=False, offset=1.0, dtype="bf16"),
        # an odd batch of odd rows, normalised with the mean, a gate per channel, fp32
        dict(name="norm 1001 rows f32", op="norm", rows=1001, dim=2559, kind="layer", post=True, gate="channel", scale=0.5, quantise=False, offset=0.0, dtype="f32"),
        # short rows in fp16, every element with a gate of its own
        dict(name="norm 3000 short rows f16", op="norm", rows=3000, dim=768, kind="rms", post=False, gate="element", scale=0.22, quantise=False, offset=0.0, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["route", "experts", "experts", "norm"])
    if op == "route":
        experts, groups = rng.choice([(8, 1), (60, 1), (64, 1), (64, 8), (128, 1), (160, 8), (256, 8), (256, 1), (384, 1), (512, 16)])
        top_groups = rng.randint(1, groups)
        top_k = min(rng.randint(1, 10), top_groups * (experts // groups))
        return dict(op=op, tokens=_log(rng, 1, 8192), experts=experts, top_k=top_k, score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups, top_groups=top_groups,
                    renormalise=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]), dtype=rng.choice(["f32", "f32", "bf16", "f16"]))
    if op == "norm":
        quantise = rng.random() < 0.3
        dim = 32 * _log(rng, 2, 256) if quantise else _log(rng, 64, 8192)
        return dict(op=op, rows=_log(rng, 1, 8192), dim=dim, kind=rng.choice(["rms", "rms", "layer"]), post=rng.random() < 0.5, gate=rng.choice(["none", "none", "row", "channel", "element"]),
                    scale=rng.choice([1.0, 0.22]), quantise=quantise, offset=rng.choice([0.0, 1.0]), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    experts = rng.choice([4, 8, 16, 60, 64, 128])
    hidden = 32 * _log(rng, 8, 160)
    inter = 32 * _log(rng, 4, min(256, (1 << 24) // (experts * hidden)))
    most = max(16, min(8192, (1 << 36) // (hidden * inter)))
    return dict(op=op, tokens=_log(rng, 1, most), experts=experts, top_k=rng.randint(1, min(8, experts)), hidden=hidden, inter=inter, act=rng.choice(["silu", "silu", "gelu"]),
                dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), skew=rng.choice([0.0, 0.5, 1.5]))


def work(case):
    el = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "route":
        return {"bytes": case["tokens"] * (case["experts"] * el + 12 * case["top_k"]) + 8 * case["experts"], "flops": 10 * case["tokens"] * case["experts"]}
    if case["op"] == "norm":
        values = case["rows"] * case["dim"]
        once = (35 / 64 if case["quantise"] else el) + 3 * el + (el if case["gate"] == "element" else 0)
        return {"bytes": int(values * once), "flops": values * (16 if case["post"] else 10)}
    t, e, k, products = case["tokens"], case["experts"], case["top_k"], 3 * case["hidden"] * case["inter"]
    met = e * (1 - (1 - k / e) ** t)
    return {"bytes": int(met * products * 35 / 64 + t * case["hidden"] * (el + 2)), "flops": 2 * t * k * products}


# ---- the format in plain torch -----------------------------------------------------------------------------------------


def _encode(x):
    """Two-stage rule along the last axis (32 elements, fp32): (index, negative, id, e + 127), every step exact."""
    book = torch.tensor(BOOK, dtype=torch.int16, device=x.device)
    top = x.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(min=-127)
    q5 = torch.floor(torch.ldexp(x.abs(), 2 - e[..., None])).to(torch.int16)
    pair = (15 - ((q5.amax(-1) + 1) // 2).clamp(max=15)).clamp(max=7).long()
    even, odd = book[2 * pair], book[2 * pair + 1]
    de, do, v5, mx = even[..., 6:7], odd[..., 6:7], even[..., 5:6], even[..., 7:8]
    in_even = ((q5 >= de + do) & (q5 < de + mx)).sum(-1)
    in_odd = ((q5 >= do + v5) & (q5 < de + do)).sum(-1)
    ids = 2 * pair + (in_odd > in_even)
    mine = (book[:, :-1] + book[:, 1:])[ids]
    index = (q5[..., None] >= mine[..., None, :]).sum(-1, dtype=torch.uint8) if x.numel() < 1 << 22 else sum((q5 >= mine[..., k : k + 1]).to(torch.uint8) for k in range(7))
    return index, torch.signbit(x), ids.to(torch.uint8), (e + 127).to(torch.uint8)


def _decode(index, negative, ids, scales):
    """fp32 values of blocks [..., 32]."""
    book = torch.tensor(BOOK, dtype=torch.float32, device=index.device).reshape(-1)
    h = book[ids.to(torch.int32)[..., None] * 8 + index.to(torch.int32)]
    return torch.ldexp(torch.where(negative, -h, h), scales.to(torch.int32)[..., None] - 128)


def _rounded(x):
    """The values that x [..., K] (fp32) has as a DialectFP4 operand."""
    return _decode(*_encode(x.unflatten(-1, (-1, 32)))).flatten(-2)


def _atoms(x):
    """One byte per (row, block) of an operand, [rows, blocks] -> [groups of 4 blocks, tiles, 32, 4, 4], zeros where there is none."""
    r, b = x.shape
    padded = torch.zeros(-(-r // 128) * 128, -(-b // 4) * 4, dtype=torch.uint8, device=x.device)
    padded[:r, :b] = x
    return padded.view(-1, 4, 32, padded.shape[1] // 4, 4).permute(3, 0, 2, 1, 4).contiguous()


def _stored(w):
    """An operand [rows, K] (fp32) as the library stores it: bytes of codes, ids, scales."""
    index, negative, ids, scales = _encode(w.view(w.shape[0], -1, 32))
    index, negative = index.view(-1, 8), negative.view(-1, 8).to(torch.uint8)
    codes = index[:, 0::2] | index[:, 1::2] << 4 | negative[:, 4:] << 3 | negative[:, :4] << 7
    i = _atoms(ids)
    return codes.reshape(-1), (i[..., 0::2] | i[..., 1::2] << 4).reshape(-1), _atoms(scales).reshape(-1)


def _values(codes, ids, scales, rows, k):
    """fp32 values [experts, rows, K] of a stack of stored operands."""
    n, nb = codes.shape[0], k // 32
    c = codes.view(n, rows, nb, 4, 4)
    index = torch.stack([c & 7, c >> 4 & 7], -1).view(n, rows, nb, 32)
    negative = torch.cat([c >> 7, c >> 3 & 1], -1).view(n, rows, nb, 32).bool()
    by_row = lambda x: x.permute(0, 2, 4, 3, 1, 5).reshape(n, -1, x.shape[1] * 4)[:, :rows, :nb]  # noqa: E731
    tiles = -(-rows // 128)
    i = ids.view(n, -1, tiles, 32, 4, 2)
    return _decode(index, negative, by_row(torch.stack([i & 15, i >> 4], -1).flatten(-2)), by_row(scales.view(n, -1, tiles, 32, 4, 4))).view(n, rows, k)


# ---- the state a program has in hand ------------------------------------------------------------------------------------


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = TYPES[case["dtype"]]
    randn = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    if case["op"] == "route":
        t, e = case["tokens"], case["experts"]
        logits = (randn(t, e) * 1.5 + 0.5 * randn(e)).to(dt)
        return dict(case=case, logits=logits, bias=0.1 * randn(e) if case["bias"] else None)
    if case["op"] == "norm":
        r, d = case["rows"], case["dim"]
        near = lambda *s: (1 + 0.2 * randn(*s) - case["offset"]).to(dt)  # noqa: E731
        channel = torch.where(torch.rand(d, generator=g, device=dev) < 0.01, 20.0, 1.0)  # outlier channels, as residual streams have them
        s = dict(case=case, y=randn(r, d).to(dt), residual=(randn(r, d) * channel * 3).to(dt), weight=near(d), post=near(d) if case["post"] else None)
        s["bias"], s["post_bias"] = ((0.1 * randn(d)).to(dt) if case["kind"] == "layer" and want else None for want in (True, case["post"]))
        gate = {"none": None, "row": (r, 1), "channel": (1, d), "element": (r, d)}[case["gate"]]
        s["gate"] = None if gate is None else torch.sigmoid(randn(*gate)).to(dt)
        return s
    t, e, k, hidden, inter = case["tokens"], case["experts"], case["top_k"], case["hidden"], case["inter"]
    channel = torch.where(torch.rand(hidden, generator=g, device=dev) < 0.01, 10.0, 1.0)
    x = (randn(t, hidden) * channel).to(dt)
    score = torch.softmax(randn(t, e) + case["skew"] * randn(e), -1)
    weights, ids = torch.topk(score, k)
    weights = weights / weights.sum(-1, keepdim=True)

    def stack(rows, cols):
        parts = [[], [], []]
        for _ in range(e):
            w = randn(rows, cols) * (cols**-0.5 * torch.exp2(randn(rows, 1) * 0.3))
            for p, x in zip(parts, _stored(w)):
                p.append(x)
        return [torch.stack(p) for p in parts]

    s = dict(case=case, x=x, ids=ids.to(torch.int32), weights=weights, up=stack(2 * inter, hidden), down=stack(hidden, inter))
    s["most"] = int(torch.bincount(ids.reshape(-1), minlength=e).max())  # rows of the busiest expert
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------


def run(s):
    return {"route": _run_route, "experts": _run_experts, "norm": _run_norm}[s["case"]["op"]](s)


def _places(ids, experts):
    """(count, place) of assignments ids [T, k]: stable order by expert, starts at multiples of 128."""
    flat = ids.reshape(-1).long()
    order = torch.sort(flat, stable=True)[1]
    count = torch.zeros(experts, dtype=torch.int64, device=ids.device).scatter_add_(0, flat, torch.ones_like(flat))
    padded = (count + 127) // 128 * 128
    start, first = padded.cumsum(0) - padded, count.cumsum(0) - count
    place = torch.empty_like(flat)
    mine = flat[order]
    place[order] = start[mine] + torch.arange(flat.numel(), device=ids.device) - first[mine]
    return count, place.view_as(ids), start


def _run_route(s):
    c = s["case"]
    if own:
        import paper_2501_01144_b200 as bd

        ids, weights, plan = bd.route(s["logits"], c["top_k"], score=c["score"], bias=s["bias"], groups=c["groups"], top_groups=c["top_groups"], renormalise=c["renormalise"], scale=c["scale"])
        return ids, weights, plan.count, plan.place
    x = s["logits"].double()  # in 64 bits: which experts are chosen hangs on the last bits of keys that lie close together
    score = torch.exp(x - x.amax(-1, keepdim=True)) if c["score"] == "softmax" else 1 / (1 + torch.exp(-x))
    if c["score"] == "softmax":
        score = score / score.sum(-1, keepdim=True)
    key = x if s["bias"] is None else score + s["bias"].double()
    if c["groups"] > 1:
        of_group = (score if s["bias"] is None else key).unflatten(-1, (c["groups"], -1))
        value = torch.sort(of_group, -1, descending=True)[0][..., :2].sum(-1)
        kept = torch.sort(value, dim=-1, descending=True, stable=True)[1][:, : c["top_groups"]]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(-1, kept, True)
        key = torch.where(keep[..., None], key.unflatten(-1, (c["groups"], -1)), float("-inf")).flatten(-2)
    ids = torch.sort(key, dim=-1, descending=True, stable=True)[1][:, : c["top_k"]]
    w = torch.gather(score, -1, ids)
    if c["renormalise"]:
        w = w / w.sum(-1, keepdim=True)
    count, place, _ = _places(ids, c["experts"])
    return ids.to(torch.int32), (w * c["scale"]).float(), count.to(torch.int32), place.to(torch.int32)


def _activate(x, act):
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return 0.5 * x * (1 + torch.tanh(0.7978845608028654 * (x + 0.044715 * x * x * x)))


def _run_experts(s):
    c = s["case"]
    e, hidden, inter, k = c["experts"], c["hidden"], c["inter"], c["top_k"]
    if own:
        import paper_2501_01144_b200 as bd

        plan = bd.expert_plan(s["ids"], e)
        up = bd.ExpertWeights.from_buffers(*s["up"], 2 * inter, hidden)
        down = bd.ExpertWeights.from_buffers(*s["down"], hidden, inter)
        return bd.expert_mlp(s["x"], plan, s["weights"], up, down, activation=c["act"], dtype=torch.bfloat16)
    _, place, start = _places(s["ids"], e)
    flat = s["ids"].reshape(-1).long()
    at = flat * s["most"] + (place.reshape(-1) - start[flat])  # row among `most` rows per expert
    x = _rounded(s["x"].float())
    rows = torch.zeros(e * s["most"], hidden, device=x.device)
    rows[at] = x.repeat_interleave(k, 0)
    u = rows.view(e, -1, hidden) @ _values(*s["up"], 2 * inter, hidden).transpose(1, 2)
    u = u.unflatten(-1, (-1, 2, 32))
    h = _rounded((_activate(u[..., 0, :], c["act"]) * u[..., 1, :]).flatten(-2))
    del u
    y = (h @ _values(*s["down"], hidden, inter).transpose(1, 2)).view(-1, hidden)[at]
    return (y.view(-1, k, hidden) * s["weights"][..., None]).sum(1).to(torch.bfloat16)


def _run_norm(s):
    c = s["case"]
    if own:
        import paper_2501_01144_b200 as bd

        h, n = bd.residual_norm(s["y"], s["weight"], s["residual"], bias=s["bias"], post_weight=s["post"], post_bias=s["post_bias"], gate=s["gate"], scale=c["scale"], norm=c["kind"], eps=1e-6,
                                weight_offset=c["offset"], quantise=c["quantise"])
        return h, bd.dequantize(n).to(torch.bfloat16) if c["quantise"] else n

    def norm(x, w, b):
        if c["kind"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * (w.float() + c["offset"])
        return x if b is None else x + b.float()

    u = s["y"].float()
    if c["post"]:
        u = norm(u, s["post"], s["post_bias"])
    if s["gate"] is not None:
        u = u * s["gate"].float()
    h = s["residual"].float() + c["scale"] * u
    n = norm(h, s["weight"], s["bias"]).to(s["y"].dtype)
    return h.to(s["y"].dtype), _rounded(n.float()).to(torch.bfloat16) if c["quantise"] else n


# ---- the same from the definitions, in 64 bits -------------------------------------------------------------------------------


def _nearest(block):
    """A block [..., 32] rounded onto its dialect's grid, from the rule's real-number form in 64 bits."""
    x = block.double()
    a = x.abs()
    top = a.amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0**-125))) - 2
    e = torch.where(top >= torch.exp2(e + 3), e + 1, torch.where(top < torch.exp2(e + 2), e - 1, e)).clamp(min=-127)
    y = a * torch.exp2(-e)
    limit = (torch.floor(2 * y.amax(-1, keepdim=True) + 0.5) / 2).clamp(max=7.5)
    book = torch.tensor(BOOK, dtype=torch.float64, device=x.device) / 2
    pair = ((7.5 - limit) * 2).clamp(max=7).long()[..., 0]
    hi, lo = book[2 * pair], book[2 * pair + 1]
    border = (hi[..., 6:7] + lo[..., 6:7]) / 2
    n_hi = ((y >= border) & (y < (hi[..., 6:7] + hi[..., 7:8]) / 2)).sum(-1)
    n_lo = ((y >= (lo[..., 6:7] + lo[..., 5:6]) / 2) & (y < border)).sum(-1)
    grid = torch.where((n_lo > n_hi)[..., None], lo, hi)
    best, off = torch.zeros_like(y), torch.full_like(y, float("inf"))
    for k in range(8):  # the larger of two equally near ones stays
        far = (y - grid[..., k : k + 1]).abs()
        best = torch.where(far <= off, grid[..., k : k + 1], best)
        off = torch.minimum(off, far)
    return torch.copysign(best, x) * torch.exp2(e)


def _nearest_rows(x):
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    per = max(1, (1 << 24) // x.shape[-1])
    for at in range(0, x.shape[0], per):
        out[at : at + per] = _nearest(x[at : at + per].unflatten(-1, (-1, 32))).flatten(-2)
    return out


def _expert(codes, ids, scales, rows, k):
    """64-bit values [rows, K] of one stored operand, byte by byte from the description of the storage."""
    dev = codes.device
    r, el = torch.arange(rows, device=dev)[:, None], torch.arange(k, device=dev)[None]
    b, j = el // 32, el % 8
    byte = r * (k // 2) + el // 8 * 4
    index = codes[byte + j // 2].long() >> (4 * (j % 2)) & 7
    sign = codes[byte + j % 4].long() >> torch.where(j < 4, 7, 3) & 1
    atom = b // 4 * (-(-rows // 128)) + r // 128
    row = r % 128
    ident = ids[atom * 256 + row % 32 * 8 + row // 32 * 2 + b % 4 // 2].long() >> (4 * (b % 2)) & 15
    scale = scales[atom * 512 + row % 32 * 16 + row // 32 * 4 + b % 4].double()
    h = torch.tensor(BOOK, dtype=torch.float64, device=dev).view(-1)[ident * 8 + index]
    return torch.where(sign == 1, -h, h) * torch.exp2(scale - 128)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        x = s["logits"].double()
        p = torch.softmax(x, -1) if case["score"] == "softmax" else torch.sigmoid(x)
        key = p if s["bias"] is None else p + s["bias"].double()
        rank = x if s["bias"] is None else key
        n, t = case["experts"] // case["groups"], x.shape[0]
        if case["groups"] > 1:
            value = torch.stack([key[:, n * j : n * j + n].topk(2, -1)[0].sum(-1) for j in range(case["groups"])], -1)
            for j in range(case["groups"]):
                ahead = (value > value[:, j : j + 1]).sum(-1) + (value[:, :j] == value[:, j : j + 1]).sum(-1)
                rank = rank.clone()
                rank[:, n * j : n * j + n][ahead >= case["top_groups"]] = float("-inf")
        picked = []
        for _ in range(case["top_k"]):
            best = rank.max(-1, keepdim=True)[0]
            which = (rank == best).to(torch.uint8).argmax(-1, keepdim=True)
            picked.append(which)
            rank = rank.scatter(-1, which, float("-inf"))
        w = torch.cat([p.gather(-1, i) for i in picked], -1)
        if case["renormalise"]:
            w = w / w.sum(-1, keepdim=True)
        return None, w * case["scale"], None, None
    if case["op"] == "norm":
        def norm(x, w, b):
            if case["kind"] == "layer":
                x = x - x.sum(-1, keepdim=True) / case["dim"]
            y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + 1e-6) * (w.double() + case["offset"])
            return y if b is None else y + b.double()

        u = s["y"].double() if s["post"] is None else norm(s["y"].double(), s["post"], s["post_bias"])
        h = s["residual"].double() + case["scale"] * (u if s["gate"] is None else u * s["gate"].double())
        n = norm(h, s["weight"], s["bias"])
        return h, _nearest_rows(n.to(s["y"].dtype)) if case["quantise"] else n
    hidden, inter = case["hidden"], case["inter"]
    x, out = _nearest_rows(s["x"].double()), torch.zeros(case["tokens"], hidden, dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        token, slot = torch.nonzero(s["ids"] == e, as_tuple=True)
        if not token.numel():
            continue
        w = _expert(*(p[e] for p in s["up"]), 2 * inter, hidden)
        u = x[token] @ w.T
        row = torch.arange(inter, device="cuda")
        gate, up = u[:, row // 32 * 64 + row % 32], u[:, row // 32 * 64 + 32 + row % 32]
        act = gate * torch.sigmoid(gate) if case["act"] == "silu" else gate * torch.sigmoid(2 * 0.7978845608028654 * (gate + 0.044715 * gate**3))
        h = _nearest_rows(act * up)
        out.index_add_(0, token, (h @ _expert(*(p[e] for p in s["down"]), hidden, inter).T) * s["weights"][token, slot].double()[:, None])
    return out
