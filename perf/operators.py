"""The operators of a serving step around the paged DialectFP4 cache, their plain forms and the cases they are timed on.

  rotate     normalisation of queries and keys per head and the position rotation, in one pass;
  cache      the step's keys and values written into the paged cache in 4 bits, and a range of it read back;
  attention  the step's queries (one token, a few, or a chunk of a prompt per sequence) against the paged cache.

`run` computes an operator from what `prepare` made: in plain torch operations, or (own = True) by the library's calls.

Storage.  A chunk is 32 tokens of one KV head, a record of 35 * d bytes.  Its keys are d / 32 tiles of 32 rows (tokens) x 32
dimensions, its values d / 32 tiles of 32 rows (channels) x 32 tokens; a row of a tile is one block (scale e + 127, 4-bit dialect
id, 32 codes).  With r = 8 j + g the row and b the tile: word t (elements 8 t .. 8 t + 7) at 4 * (((8 b + g) * 4 + t) * 4 + j),
scale byte at (4 g + j) * (d / 32) + b, id nibble at the same index.  Row of token 8 x + 2 y + z in a key tile: 8 y + 2 x + z.
Parts of a record: key codes, value codes (16 d each), key scales, value scales (d each), key ids, value ids (d / 2 each).
Elements 0 .. 7 of a word sit in its nibbles 0, 2, 1, 3, 4, 6, 5, 7 as sign << 3 | index.  The values of an unfinished chunk are
rows token % 64 of the sequence's tail, in the source type.
"""
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# The DialectFP4 formatbook in units of 0.5: pair p has the maximum 15 - p, and its members differ in their second largest value.
_SECOND = ((12, 10), (11, 9), (10, 8), (9, 8), (9, 8), (8, 7), (8, 7), (7, 6))
BOOK = [[0, 1, 2, 3, 4, 5 if p == 7 else 6, _SECOND[p][o], 15 - p] for p in range(8) for o in range(2)]
NIBBLE = (0, 2, 1, 3, 4, 6, 5, 7)


# ---- the cases ------------------------------------------------------------------------------------------------------


def listed():
    return [
        # one decode step of 64 sequences: rows of a fused projection, latency
        dict(name="rotate 64 rows", op="rotate", rows=64, heads=32, kv_heads=8, dim=128, rot=128, dtype="bf16", norm=True, pairs="halves"),
        # a prefill batch of 8192 tokens
        dict(name="rotate 8192 rows", op="rotate", rows=8192, heads=32, kv_heads=8, dim=128, rot=128, dtype="bf16", norm=True, pairs="halves"),
        # an odd batch of a small model: a part of each head rotated, neighbouring pairs, no normalisation
        dict(name="rotate 1001 rows f32", op="rotate", rows=1001, heads=32, kv_heads=32, dim=64, rot=32, dtype="f32", norm=False, pairs="neighbours"),
        # one decode step of 64 sequences written, the last tokens of each read back
        dict(name="cache step of 64", op="cache", n=64, new_min=1, new_max=1, old_min=0, old_max=4096, old_unit=1, read=64, kv_heads=8, dim=128, page=64, dtype="bf16", salt=1),
        # prompts of ragged lengths written from empty and read back whole
        dict(name="cache prompts", op="cache", n=7, new_min=600, new_max=1700, old_min=0, old_max=0, old_unit=32, read=8192, kv_heads=8, dim=128, page=64, dtype="bf16", salt=2),
        # a few tokens a sequence (drafts to be verified), small heads, fp16
        dict(name="cache drafts f16", op="cache", n=33, new_min=1, new_max=7, old_min=0, old_max=1000, old_unit=1, read=100, kv_heads=32, dim=64, page=32, dtype="f16", salt=3),
        # one sequence, one token: latency
        dict(name="attention 1 x 513", op="attention", n=1, new_min=1, new_max=1, kv_min=513, kv_max=513, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", softcap=0.0, window=0, salt=4),
        # an ordinary decode batch
        dict(name="attention 32 x 4113", op="attention", n=32, new_min=1, new_max=1, kv_min=1500, kv_max=4113, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", softcap=0.0, window=0, salt=5),
        # a full decode batch of long contexts
        dict(name="attention 64 x 12000", op="attention", n=64, new_min=1, new_max=1, kv_min=6000, kv_max=12000, heads=32, kv_heads=8, dim=128, page=128, dtype="bf16", softcap=0.0, window=0, salt=6),
        # drafts of up to four tokens verified, capped scores, a sliding window
        dict(name="attention drafts capped", op="attention", n=48, new_min=1, new_max=4, kv_min=5, kv_max=3000, heads=32, kv_heads=8, dim=128, page=32, dtype="bf16", softcap=30.0, window=1024, salt=7),
        # chunks of several prompts over what each has so far, small heads, fp16
        dict(name="attention chunks f16", op="attention", n=6, new_min=1, new_max=700, kv_min=700, kv_max=4096, heads=32, kv_heads=32, dim=64, page=64, dtype="f16", softcap=0.0, window=0, salt=8),
        # a long prompt's last chunk of 4096 tokens
        dict(name="attention 4096 of 16384", op="attention", n=1, new_min=4096, new_max=4096, kv_min=16384, kv_max=16384, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16", softcap=0.0, window=0, salt=9),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["rotate", "cache", "attention", "attention"])
    heads, kv_heads = rng.choice([(32, 8), (32, 32), (16, 2), (28, 4), (8, 8), (24, 8)])
    dim = rng.choice([64, 128])
    if op == "rotate":
        return dict(op=op, rows=_log(rng, 1, 8192), heads=heads, kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim, dim // 2]), dtype=rng.choice(["bf16", "bf16", "f16"]), norm=rng.random() < 0.7,
                    pairs=rng.choice(["halves", "neighbours"]))
    page, salt = rng.choice([32, 64, 128]), rng.randrange(1 << 20)
    if op == "cache":
        n = _log(rng, 1, 64)
        prompt = rng.random() < 0.5
        new = _log(rng, 33, max(33, 8192 // n)) if prompt else rng.randint(1, 8)
        return dict(op=op, n=n, new_min=1 + new // 3, new_max=new, old_min=0, old_max=rng.randint(0, 3000), old_unit=32 if prompt else 1, read=_log(rng, 1, 4096), kv_heads=kv_heads, dim=dim, page=page,
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), salt=salt)
    more = dict(heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=rng.choice(["bf16", "bf16", "f16"]), softcap=rng.choice([0.0, 0.0, 30.0, 50.0]), window=rng.choice([0, 0, _log(rng, 1, 4096)]), salt=salt)
    if rng.random() < 0.6:
        n = _log(rng, 1, 64)
        kv = _log(rng, 1, 12000 if kv_heads <= 8 else 4000)
        return dict(op=op, n=n, new_min=1, new_max=rng.choice([1, 1, 2, 5]), kv_min=max(1, kv // 3), kv_max=kv, **more)
    n, new = rng.randint(1, 6), _log(rng, 6, 1500)
    return dict(op=op, n=n, new_min=1 + new // 2, new_max=new, kv_min=new, kv_max=new + _log(rng, 1, 6000), **more)


def _lengths(case):
    """(tokens of the step, tokens in the cache after it) of each sequence."""
    rng = random.Random(case["salt"])
    new, total = [], []
    for k in range(case["n"]):
        t = rng.randint(case["new_min"], case["new_max"])
        if case["op"] == "cache":
            u = case["old_unit"]
            total.append(t + u * rng.randint(-(-case["old_min"] // u), case["old_max"] // u))
        else:
            total.append(max(t, case["kv_max"] if k == 0 else rng.randint(case["kv_min"], case["kv_max"])))
        new.append(t)
    return new, total


def work(case):
    el = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotate":
        values = case["rows"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * el * values + case["rows"] * (4 * case["rot"] + 4) + (2 * case["dim"] * el if case["norm"] else 0), "flops": 7 * values}
    new, total = _lengths(case)
    per_token = 2 * case["kv_heads"] * case["dim"]  # key and value elements
    packed = 35 / 64
    if case["op"] == "cache":
        back = sum(min(case["read"], t) for t in total)
        return {"bytes": int(per_token * (sum(new) * (el + packed) + back * (packed + el))), "flops": 10 * per_token * (sum(new) + back)}
    seen = kept = 0
    for t, m in zip(new, total):
        w = case["window"] or m
        seen += sum(min(w, m - t + i + 1) for i in range(t))
        kept += min(m, w + t - 1)
    rows = sum(new) * case["heads"] * case["dim"]
    return {"bytes": int(per_token * packed * kept + 2 * el * rows), "flops": 4 * seen * case["heads"] * case["dim"]}


# ---- the format in plain torch -----------------------------------------------------------------------------------------


def _encode(x):
    """Two-stage rule along the last axis (32 elements, fp32): (code = sign << 3 | index, id, e + 127), every step exact."""
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
    steps = book[:, :-1] + book[:, 1:]
    index = torch.zeros_like(q5, dtype=torch.uint8)
    mine = steps[ids]
    for k in range(7):
        index += q5 >= mine[..., k : k + 1]
    return index + 8 * torch.signbit(x).to(torch.uint8), ids.to(torch.uint8), (e + 127).to(torch.uint8)


def _decode(codes, ids, scales):
    """fp32 values of codes [..., 32]; ids and scales [...]."""
    book = torch.tensor(BOOK, dtype=torch.float32, device=codes.device).reshape(-1)
    signed = torch.cat([book.view(16, 8), -book.view(16, 8)], 1).reshape(-1)
    h = signed[ids.to(torch.int32)[..., None] * 16 + codes.to(torch.int32)]
    return torch.ldexp(h, scales.to(torch.int32)[..., None] - 128)


def _pack(codes, ids, scales):
    """One operand's tiles: codes [m, tiles, 32 rows, 32], ids and scales [m, tiles, 32] -> bytes of codes, scales, ids."""
    m, nb = codes.shape[:2]
    w = codes.view(m, nb, 4, 8, 4, 8).permute(0, 1, 3, 4, 2, 5)  # tile, g, word, j, element
    where = [NIBBLE.index(k) for k in range(8)]
    w = w[..., where]
    packed = (w[..., 0::2] | w[..., 1::2] << 4).reshape(m, -1)
    by_row = lambda x: x.view(m, nb, 4, 8).permute(0, 3, 2, 1).reshape(m, -1)  # noqa: E731  (g, j, tile)
    i = by_row(ids)
    return packed, by_row(scales).contiguous(), i[:, 0::2] | i[:, 1::2] << 4


def _unpack(packed, scales, ids, nb):
    """The inverse of _pack."""
    m = packed.shape[0]
    both = torch.stack([packed & 15, packed >> 4], -1).view(m, nb, 8, 4, 4, 8)[..., list(NIBBLE)]
    codes = both.permute(0, 1, 4, 2, 3, 5).reshape(m, nb, 32, 32)
    by_tile = lambda x: x.view(m, 8, 4, nb).permute(0, 3, 2, 1).reshape(m, nb, 32)  # noqa: E731
    return codes, by_tile(torch.stack([ids & 15, ids >> 4], -1).view(m, -1)), by_tile(scales)


def _to_rows(x):
    """[m, 32 tokens, ...] -> the rows of a key tile."""
    return x.unflatten(1, (4, 4, 2)).transpose(1, 2).flatten(1, 3)


_to_tokens = _to_rows  # the exchange of the two halves of the index is its own inverse


def _records(k, v):
    """Whole chunks: keys and values [m, 32, d] in any type -> records [m, 35 d]."""
    m, _, d = k.shape
    kc, ki, ks = _encode(k.float().view(m, 32, d // 32, 32))
    vc, vi, vs = _encode(v.float().transpose(1, 2).reshape(m, d // 32, 32, 32))
    kc, ki, ks = (_to_rows(x).transpose(1, 2) for x in (kc, ki, ks))
    a, b, c = _pack(kc.contiguous(), ki.contiguous(), ks.contiguous())
    p, q, r = _pack(vc, vi, vs)
    return torch.cat([a, p, b, q, c, r], 1)


def _chunks(records, d):
    """Records [m, 35 d] -> fp32 keys and values [m, 32, d]."""
    m, nb = records.shape[0], d // 32
    a, p, b, q, c, r = torch.split(records, [16 * d, 16 * d, d, d, d // 2, d // 2], 1)
    k = _decode(*_unpack(a.contiguous(), b.contiguous(), c.contiguous(), nb))
    v = _decode(*_unpack(p.contiguous(), q.contiguous(), r.contiguous(), nb))
    return _to_tokens(k.transpose(1, 2)).reshape(m, 32, d), v.reshape(m, d, 32).transpose(1, 2)


def _in_parts(f, n, size, out):
    for at in range(0, n, size):
        out[at : at + size] = f(at, min(n, at + size))
    return out


# ---- the state a serving program has in hand ------------------------------------------------------------------------------


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    dt, d = TYPES[case["dtype"]], case["dim"]
    randn = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    if case["op"] == "rotate":
        rows, h, hk, rot = case["rows"], case["heads"], case["kv_heads"], case["rot"]
        qkv = (randn(rows, (h + 2 * hk) * d) * 2).to(dt)  # the fused projection's result
        angle = torch.arange(16384, device=dev, dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        table = torch.cat([angle.cos(), angle.sin()], 1).float()  # the program's table of cosines and sines
        pos = torch.randint(0, 16384, (rows,), generator=g, device=dev, dtype=torch.int32)
        weights = [(1 + 0.2 * randn(d)).to(dt) if case["norm"] else None for _ in range(2)]
        return dict(case=case, q=qkv[:, : h * d].view(rows, h, d), k=qkv[:, h * d : (h + hk) * d].view(rows, hk, d), table=table, pos=pos, wq=weights[0], wk=weights[1])
    new, total = _lengths(case)
    n, hk, page = case["n"], case["kv_heads"], case["page"]
    per_page = page // 32
    width = max(-(-t // page) for t in total)
    pages = sum(-(-t // page) for t in total) + 3
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table = torch.zeros(n, width, dtype=torch.int32, device=dev)
    at = 0
    for i, t in enumerate(total):
        used = -(-t // page)
        table[i, :used] = order[at : at + used]
        at += used
    channel = torch.where(torch.rand(hk, d, generator=g, device=dev) < 0.02, 6.0, 1.0)  # outlier channels, as keys have them
    spread = torch.exp2(torch.randint(-2, 3, (hk, d), generator=g, device=dev).float())

    def rows_of(m):
        return (randn(m, hk, d) * channel).to(dt), (randn(m, hk, d) * spread).to(dt)

    # the tokens that earlier steps stored (for the attention: this step's too)
    pool = torch.zeros(pages, hk, per_page, 35 * d, dtype=torch.uint8, device=dev)
    flat = pool.view(-1, 35 * d)
    tail = torch.zeros(n + 2, hk, 64, d, dtype=dt, device=dev)
    slots = torch.randperm(n + 2, generator=g, device=dev)[:n].to(torch.int32)
    stored = total if case["op"] == "attention" else [m - t for t, m in zip(new, total)]
    per = max(1, (1 << 24) // (hk * d * 32))  # chunks a turn
    for i, m in enumerate(stored):
        full = m // 32
        for c0 in range(0, -(-m // 32), per):
            c1 = min(-(-m // 32), c0 + per)
            k, v = rows_of(32 * (c1 - c0))
            rec = _records(k.view(-1, 32, hk, d).transpose(1, 2).reshape(-1, 32, d), v.view(-1, 32, hk, d).transpose(1, 2).reshape(-1, 32, d)).view(-1, hk, 35 * d)
            c = torch.arange(c0, c1, device=dev)
            where = (table[i, c // per_page].long()[:, None] * hk + torch.arange(hk, device=dev)) * per_page + (c % per_page)[:, None]
            flat[where.reshape(-1)] = rec.reshape(-1, 35 * d)
            if c1 > full:
                at32 = 32 * (full % 2)
                tail[slots[i].long(), :, at32 : at32 + m % 32] = v[32 * (full - c0) : 32 * (full - c0) + m % 32].transpose(0, 1)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    starts = lambda x: ints([sum(x[:i]) for i in range(len(x) + 1)])  # noqa: E731
    s = dict(case=case, pool=pool, tail=tail, table=table, slots=slots, kv_len=ints(total), q_start=starts(new), rows=sum(new), max_new=max(new))
    if case["op"] == "cache":
        back = [min(case["read"], t) for t in total]
        s["k"], s["v"] = rows_of(sum(new))
        s.update(r_start=starts(back), back=sum(back), max_back=max(back))
    else:
        s["q"] = randn(sum(new), case["heads"], d).to(dt)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------


def run(s):
    return {"rotate": _run_rotate, "cache": _run_cache, "attention": _run_attention}[s["case"]["op"]](s)


def _batch(s):
    import paper_2501_01144_b200 as bd

    cache = bd.PagedKVCache.from_buffers(s["pool"], s["tail"], s["case"]["page"])
    return bd, cache, bd.PagedBatch(s["table"], s["slots"], s["kv_len"], s["q_start"], s["max_new"])


def _run_rotate(s):
    c = s["case"]
    if own:
        import paper_2501_01144_b200 as bd

        return bd.qk_norm_rope(s["q"], s["k"], s["pos"], s["table"], s["wq"], s["wk"], eps=1e-6, interleaved=c["pairs"] == "neighbours")
    rot = c["rot"]
    at = s["table"][s["pos"].long()]
    cos, sin = at[:, None, : rot // 2], at[:, None, rot // 2 :]

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        a, b = (y[..., : rot // 2], y[..., rot // 2 : rot]) if c["pairs"] == "halves" else (y[..., 0:rot:2], y[..., 1:rot:2])
        u, v = a * cos - b * sin, b * cos + a * sin
        turned = torch.cat([u, v], -1) if c["pairs"] == "halves" else torch.stack([u, v], -1).flatten(-2)
        return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)

    return one(s["q"], s["wq"]), one(s["k"], s["wk"])


def _positions(kv_len, start, most, dev):
    """Rows and tokens of the last start[i + 1] - start[i] tokens of each sequence: (valid, token) [n, most]."""
    i = torch.arange(most, device=dev)[None]
    t = (start[1:] - start[:-1])[:, None]
    return i < t, kv_len[:, None] - t + i


def _run_cache(s):
    c = s["case"]
    if own:
        bd, cache, batch = _batch(s)
        bd.paged_append(cache, batch, s["k"], s["v"])
        back = bd.PagedBatch(s["table"], s["slots"], s["kv_len"], s["r_start"], s["max_back"])
        return bd.paged_read(cache, back, s["back"])
    hk, d, page, dev = c["kv_heads"], c["dim"], c["page"], s["pool"].device
    per_page, flat = page // 32, s["pool"].view(-1, 35 * c["dim"])
    heads = torch.arange(hk, device=dev)
    ok, token = _positions(s["kv_len"], s["q_start"], s["max_new"], dev)
    seq, tok = torch.arange(c["n"], device=dev)[:, None].expand_as(token)[ok], token[ok]
    old = s["kv_len"] - (s["q_start"][1:] - s["q_start"][:-1])
    # every chunk that the step touches, as 32 source rows: the waiting rows of the tail, then the new ones
    first = old // 32
    most = (s["max_new"] + 31) // 32 + 1
    ch = first[:, None] + torch.arange(most, device=dev)[None]
    touched = ch < ((s["kv_len"] + 31) // 32)[:, None]
    src = torch.zeros(2, c["n"], most * 32, hk, d, dtype=s["k"].dtype, device=dev)
    waiting = old % 32
    lane = torch.arange(32, device=dev)
    early = s["tail"][s["slots"].long()[:, None], :, (32 * (first % 2))[:, None] + lane]
    src[1, :, :32] = torch.where((lane < waiting[:, None])[..., None, None], early, src[1, :, :32])
    at = tok - 32 * first[seq]
    src[0, seq, at], src[1, seq, at] = s["k"], s["v"]
    sel = touched.reshape(-1)
    k, v = (x.reshape(-1, 32, hk, d)[sel].transpose(1, 2).reshape(-1, 32, d) for x in src)
    fresh = _records(k, v)
    cs, cc = torch.arange(c["n"], device=dev)[:, None].expand_as(ch).reshape(-1)[sel], ch.reshape(-1)[sel]
    where = ((s["table"][cs, (cc // per_page).long()].long()[:, None] * hk + heads) * per_page + (cc % per_page)[:, None]).reshape(-1)
    # keys of earlier tokens and the values of an unfinished chunk stay as they are
    kept = flat[where]
    tokens = (32 * cc)[:, None] + lane
    is_new = (tokens >= old[cs][:, None]) & (tokens < s["kv_len"][cs][:, None])
    rows = _to_rows(is_new.view(-1, 32, 1))[..., 0].view(-1, 4, 8)  # (j, g)
    nb = d // 32
    key_word = rows.permute(0, 2, 1)[:, None, :, None, :, None].expand(-1, nb, -1, 4, -1, 4).reshape(-1, 16 * d)
    key_scale = rows.permute(0, 2, 1)[..., None].expand(-1, -1, -1, nb).reshape(-1, d)
    done = (32 * (cc + 1) <= s["kv_len"][cs])[:, None]
    mask = torch.cat([key_word, done.expand(-1, 16 * d), key_scale, done.expand(-1, d), key_scale[:, ::2], done.expand(-1, d // 2)], 1)
    flat[where] = torch.where(mask.repeat_interleave(hk, 0), fresh, kept)
    # the newest rows, and those of the chunk before, in the source type
    recent = tok >= 32 * (s["kv_len"][seq] // 32) - 32
    s["tail"][s["slots"][seq[recent]].long(), :, (tok[recent] % 64).long()] = s["v"][recent]
    k, v = _all_tokens(s)
    ok, token = _positions(s["kv_len"], s["r_start"], s["max_back"], dev)
    seq, tok = torch.arange(c["n"], device=dev)[:, None].expand_as(token)[ok], token[ok]
    return k[seq, :, tok.long()].to(s["tail"].dtype), v[seq, :, tok.long()].to(s["tail"].dtype)


def _all_tokens(s):
    """fp32 keys and values [n, heads, width * page, d] of every sequence, zeros behind its last token."""
    c = s["case"]
    n, hk, d, dev = c["n"], c["kv_heads"], c["dim"], s["pool"].device
    rec = s["pool"][s["table"].long()].permute(0, 2, 1, 3, 4).reshape(-1, 35 * d)
    m, per = rec.shape[0], (1 << 27) // (32 * d)
    k, v = (torch.empty(m, 32, d, device=dev) for _ in range(2))
    for at in range(0, m, per):
        k[at : at + per], v[at : at + per] = _chunks(rec[at : at + per], d)
    k, v = k.view(n, hk, -1, d), v.view(n, hk, -1, d)
    token = torch.arange(k.shape[2], device=dev)[None]
    k.masked_fill_((token >= s["kv_len"][:, None])[:, None, :, None], 0.0)
    v.masked_fill_((token >= 32 * (s["kv_len"] // 32)[:, None])[:, None, :, None], 0.0)
    lane = torch.arange(32, device=dev)
    at = 32 * (s["kv_len"] // 32)[:, None] + lane
    ok = at < s["kv_len"][:, None]
    seq = torch.arange(n, device=dev)[:, None].expand_as(at)[ok]
    v[seq, :, at[ok].long()] = s["tail"][s["slots"][seq].long(), :, (at[ok] % 64).long()].float()
    return k, v


def _run_attention(s):
    c = s["case"]
    if own:
        bd, cache, batch = _batch(s)
        return bd.paged_attention(cache, batch, s["q"], softcap=c["softcap"], window=c["window"])
    hk, d, dev = c["kv_heads"], c["dim"], s["pool"].device
    k, v = _all_tokens(s)
    ok, token = _positions(s["kv_len"], s["q_start"], s["max_new"], dev)
    row = (s["q_start"][:-1, None] + torch.arange(s["max_new"], device=dev)[None]).clamp(max=s["rows"] - 1).long()
    q = s["q"].float()[row].view(c["n"], s["max_new"], hk, c["heads"] // hk, d).transpose(1, 2).reshape(c["n"], hk, -1, d)
    x = q @ k.transpose(-1, -2) * d**-0.5
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    key = torch.arange(k.shape[2], device=dev)
    see = (key <= token[..., None]) & ok[..., None]
    if c["window"]:
        see &= key > token[..., None] - c["window"]
    x = x.view(c["n"], hk, s["max_new"], -1, k.shape[2])
    x.masked_fill_(~see[:, None, :, None], float("-inf"))
    x -= x.amax(-1, keepdim=True).clamp(min=-3e38)
    x.exp_()
    o = (x.flatten(2, 3) @ v).view(c["n"], hk, s["max_new"], -1, d) / x.sum(-1, keepdim=True).clamp(min=1e-38)
    return o.transpose(1, 2)[ok].reshape(-1, c["heads"], d).to(s["q"].dtype)


# ---- the same from the definitions, in 64 bits -------------------------------------------------------------------------------


def _value_of(record, d, key, token, channel):
    """Values of elements (token, channel) [m] of the records [m, 35 d], byte by byte from the description of the storage."""
    nb = d // 32
    if key:
        row, tile, el = 8 * (token // 2 % 4) + 2 * (token // 8) + token % 2, channel // 32, channel % 32
    else:
        row, tile, el = channel % 32, channel // 32, token
    g, j = row % 8, row // 8
    nib = torch.tensor(NIBBLE, device=record.device)[el % 8]
    at = (0 if key else 16 * d) + 4 * (((8 * tile + g) * 4 + el // 8) * 4 + j) + nib // 2
    pick = lambda i: torch.gather(record, -1, i).long()  # noqa: E731
    code = pick(at) >> (4 * (nib % 2)) & 15
    entry = (4 * g + j) * nb + tile
    ident = pick((34 * d if key else 34 * d + d // 2) + entry // 2) >> (4 * (entry % 2)) & 15
    scale = pick((32 * d if key else 33 * d) + entry)
    half = torch.tensor(BOOK, dtype=torch.float64, device=record.device).view(-1)[ident * 8 + (code & 7)]
    return torch.where(code >= 8, -half, half) * torch.exp2((scale - 128).double())


def _exact_sequence(s, i, pool, tail):
    """64-bit keys and values [heads, tokens, d] of sequence i."""
    c = s["case"]
    hk, d, page, m = c["kv_heads"], c["dim"], c["page"], int(s["kv_len"][i])
    dev = pool.device
    k, v = (torch.zeros(hk, m, d, dtype=torch.float64, device=dev) for _ in range(2))
    token, channel = (x.reshape(1, -1) for x in torch.meshgrid(torch.arange(32, device=dev), torch.arange(d, device=dev), indexing="ij"))
    per = 256
    for c0 in range(0, -(-m // 32), per):
        ch = torch.arange(c0, min(-(-m // 32), c0 + per), device=dev)
        rec = pool[s["table"][i, ch // (page // 32)].long(), :, ch % (page // 32)].reshape(-1, 35 * d)
        for key, out in ((True, k), (False, v)):
            x = _value_of(rec, d, key, token.expand(rec.shape[0], -1), channel.expand(rec.shape[0], -1)).view(len(ch), hk, 32, d).transpose(0, 1).reshape(hk, -1, d)
            out[:, 32 * c0 : 32 * (c0 + len(ch))] = x[:, : m - 32 * c0]
    for t in range(m // 32 * 32, m):
        v[:, t] = tail[int(s["slots"][i]), :, t % 64].double()
    return k, v


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
    off = (y[..., None] - grid[..., None, :]).abs().flip(-1)  # the larger of two equally near ones comes first
    best = torch.gather(grid[..., None, :].expand(*y.shape, 8), -1, 7 - off.argmin(-1, keepdim=True))[..., 0]
    return torch.copysign(best, x) * torch.exp2(e)


def exact(case, seed):
    s = prepare(case, seed)
    d = case["dim"]
    if case["op"] == "rotate":
        rot, out = case["rot"], []
        p, f = s["pos"].long(), s["table"].double()
        for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
            y = x.double()
            if w is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + 1e-6) * w.double()
            z = y.clone()
            for m in range(rot // 2):
                i, j = (m, m + rot // 2) if case["pairs"] == "halves" else (2 * m, 2 * m + 1)
                co, si = f[p, m][:, None], f[p, m + rot // 2][:, None]
                z[..., i], z[..., j] = y[..., i] * co - y[..., j] * si, y[..., j] * co + y[..., i] * si
            out.append(z)
        return tuple(out)
    if case["op"] == "cache":
        new, total = _lengths(case)
        ks, vs, at = [], [], 0
        for i, (t, m) in enumerate(zip(new, total)):
            old, back = m - t, min(case["read"], m)
            before = dict(s, kv_len=torch.where(torch.arange(case["n"], device="cuda") == i, old, s["kv_len"]))
            k, v = _exact_sequence(before, i, s["pool"], s["tail"])
            fresh = s["k"][at : at + t].view(t, -1, d // 32, 32)
            k = torch.cat([k, _nearest(fresh).view(t, -1, d).transpose(0, 1)], 1)
            source = torch.cat([v, s["v"][at : at + t].double().transpose(0, 1)], 1)
            for c0 in range(old // 32 * 32, m // 32 * 32, 32):
                source[:, c0 : c0 + 32] = _nearest(source[:, c0 : c0 + 32].transpose(1, 2)).transpose(1, 2)
            ks.append(k[:, m - back :].transpose(0, 1))
            vs.append(source[:, m - back :].transpose(0, 1))
            at += t
        return torch.cat(ks), torch.cat(vs)
    out = torch.zeros(s["rows"], case["heads"], d, dtype=torch.float64, device="cuda")
    new, total = _lengths(case)
    group, at = case["heads"] // case["kv_heads"], 0
    for i, (t, m) in enumerate(zip(new, total)):
        k, v = _exact_sequence(s, i, s["pool"], s["tail"])
        where = torch.arange(m - t, m, device="cuda")[:, None]
        key = torch.arange(m, device="cuda")[None]
        see = key <= where
        if case["window"]:
            see &= where - key < case["window"]
        for h in range(case["heads"]):
            x = s["q"][at : at + t, h].double() @ k[h // group].T / d**0.5
            if case["softcap"]:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            out[at : at + t, h] = torch.softmax(torch.where(see, x, float("-inf")), -1) @ v[h // group]
        at += t
    return out
