"""Attention over the paged cache at its edges: caps from far below to far above the scores, pages that are not there.  Against
64 bits, on every way a call can take."""
import numpy as np
import pytest
import torch

import paper_2501_01144_b200 as bd
from paged_util import World, source_rows, values_of
from paper_2501_01144_b200 import inputs
from util import to_device

pytestmark = pytest.mark.gpu
F16_HALF_STEP = 2.0 ** -11

# (head_dim, query heads, KV heads, tokens there, rows): which kernels serve the call
WAYS = {
    "a CTA per head": (128, 4, 2, 300, 1),
    "a CTA per head, 16 columns": (64, 8, 2, 290, 3),
    "runs and join": (64, 8, 1, 2900, 1),
    "runs and join, 16 columns": (128, 4, 1, 2900, 4),
    "row tiles": (64, 4, 2, 333, 40),
    "two row tiles": (128, 8, 2, 400, 70),
    "row tiles, shared tokens": (128, 4, 1, 4100, 33),
    "tiles expanded in front": (128, 8, 1, 6500, 520),
}


def i32(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


def bits_of(x, kind):
    x = np.asarray(x, np.float32)
    return inputs.to_bf16_bits(x) if kind == torch.bfloat16 else inputs.to_f16_bits(x)


def ask(w, q_bits, t, heads, table=None, **kw):
    """The last t tokens' rows of sequence 0 alone: fp32 output and log-sum-exp as fp64."""
    lse = torch.full((t, heads), 7.0, device="cuda")
    b = bd.PagedBatch(w.table if table is None else table, w.slots, i32([w.seqs[0].length]), i32([0, t]), t)
    o = bd.paged_attention(w.cache, b, to_device(q_bits, w.kind), dtype=torch.float32, lse=lse, **kw)
    return o.double().cpu().numpy(), lse.double().cpu().numpy()


def compare(got, q, k, v, see, scale, kind, softcap=0.0, wide=None):
    """got = (o, lse) against softmax(scores of q [t, heads, d] and k [kv_heads, n, d] where see [t, n]) v, all in fp64."""
    o, lse = got
    t, heads, d = q.shape
    group = heads // k.shape[0]
    # more than 16 rows per KV head: probabilities in the cache's type, values of fp16 caches in fp16 (half of its smallest step)
    wide = group * t > 16 if wide is None else wide
    p_half_step = 2.0 ** -8 if wide and kind == torch.bfloat16 else F16_HALF_STEP
    # fp16 probabilities: half of the smallest step, 2^-25, and the largest of a row is at least 2^7 in the kernels' units
    p_floor = 0.0 if wide and kind == torch.bfloat16 else 2.0 ** -32
    v_floor = 2.0 ** -25 if wide and kind == torch.float16 else 0.0
    for h in range(heads):
        kh, vh = k[h // group], v[h // group]
        s = scale * (q[:, h] @ kh.T)
        # exact products, at most 128 + 8 fp32 roundings of sums, each relative to the sum of the products' sizes
        ds = 136 * 2.0 ** -24 * abs(scale) * (np.abs(q[:, h]) @ np.abs(kh).T)
        if softcap:
            # c x P(x^2) / Q(x^2) with x = y / c within +-8, all coefficients positive: the fit 2^-22.6 (tanh(8) itself is 1 - 2^-22), x three
            # roundings, P and Q two each, the reciprocal and three products seven halves: 13 * 2^-24 + 2^-22.6 < 2^-20 of the result
            s = softcap * np.tanh(s / softcap)
            ds = ds + 2.0 ** -20 * np.abs(s)
        s = np.where(see, s, -np.inf)
        seen = see.any(1)
        m = np.where(seen, s.max(1), 0.0)
        p = np.exp(s - m[:, None])
        total = np.where(seen, p.sum(1), 1.0)
        ref = p @ vh / total[:, None]
        size, flat = p @ np.abs(vh) / total[:, None], see @ np.abs(vh) / total[:, None]
        # the score in units of log2 e, its difference from the reference: four roundings of the largest score's size
        dsm = np.where(see, ds, 0).max(1) + 2.0 ** -22 * np.where(see, np.abs(s), 0).max(1)
        # exp2 2^-22, sums of see.sum() terms in fp32
        rel = p_half_step + 2 * dsm + 2.0 ** -21 + see.sum(1) * 2.0 ** -24
        bound = rel[:, None] * size + p_floor * flat + v_floor + 2.0 ** -24 * np.abs(ref)
        err = np.abs(o[:, h] - ref)
        assert (err <= bound).all(), f"head {h}: error {np.nanmax(err)}, error / bound {np.nanmax(err / np.maximum(bound, 1e-300))}"
        want = m + np.log(total)
        assert (np.isinf(lse[:, h]) == ~seen).all()
        off = np.abs(np.where(seen, lse[:, h], 0) - np.where(seen, want, 0))
        assert (off <= dsm + 2.0 ** -20 + see.sum(1) * 2.0 ** -24 + 2.0 ** -23 * np.abs(want)).all(), f"head {h}: log-sum-exp off by {off.max()}"


def causal(n, t, window=0):
    key, pos = np.arange(n)[None], np.arange(n - t, n)[:, None]
    return (key <= pos) & ((key > pos - window) if window else True)


def world(way, kind, seed):
    d, heads, kv_heads, n, t = WAYS[way]
    w = World(1, kv_heads, d, 32, kind, seed=seed, max_tokens=n)
    w.step([n])
    q = bits_of(w.rng.standard_normal((t, heads, d)), kind)
    return w, q, t, heads


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("softcap", [3.0, 50.0, 1e3, 1e5, 1e8, 1e30])
def test_a_cap_costs_no_accuracy_however_far_above_the_scores(kind, way, softcap):
    w, q, t, heads = world(way, kind, seed=50)
    s = w.seqs[0]
    got = ask(w, q, t, heads, softcap=softcap)
    bd.poll_status()
    compare(got, values_of(q, kind), s.keys(), s.values(), causal(s.length, t), w.d ** -0.5, kind, softcap)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("window", [0, 270])
def test_tokens_of_a_bad_page_are_not_seen(kind, way, window):
    """Page numbers outside the pool inside the visible range: the result is that of the other tokens, although the missing ones
    have the largest scores (or, a second time, all scores are alike, so that keys left over from other tiles would count)."""
    d, heads, kv_heads, n, t = WAYS[way]
    rng = np.random.default_rng(60)
    common = rng.standard_normal(d)
    pages = -(-n // 32)
    near = (n - t - 130) // 32                                      # a page that every row's window of 270 tokens holds
    bad = {near: -1, pages - 1: 2 ** 31 - 1}                        # the last one: an unfinished chunk
    if not window:
        bad |= {0: -7, 5: None, 6: -2 ** 31} | ({k: -1 for k in range(12, 16)} if pages > 16 else {})
    token = np.arange(n)
    gone = np.isin(token // 32, list(bad))
    for loud in (True, False):
        w = World(1, kv_heads, d, 32, kind, seed=61, max_tokens=n)
        k, v = source_rows(rng, n, kv_heads, d, torch.float32)
        if loud:
            k[gone] = 0.4 * common
        else:
            k *= 0.1
        k, v = bits_of(k, kind), bits_of(v, kind)
        w.seqs[0].append(k, v)
        bd.paged_append(w.cache, w.batch([n]), to_device(k, kind), to_device(v, kind))
        q = bits_of(common + 0.5 * rng.standard_normal((t, heads, d)), kind)
        table = w.table.clone()
        for page, number in bad.items():
            table[0, page] = w.cache.pages if number is None else number
        s = w.seqs[0]
        args = values_of(q, kind), s.keys(), s.values()
        whole = ask(w, q, t, heads, window=window)
        bd.poll_status()
        compare(whole, *args, causal(n, t, window), d ** -0.5, kind)
        got = ask(w, q, t, heads, table=table, window=window)
        with pytest.raises(bd.BdError) as e:
            bd.poll_status()
        assert e.value.status == 10
        compare(got, *args, causal(n, t, window) & ~gone, d ** -0.5, kind)
        if loud:
            with pytest.raises(AssertionError):                     # the missing tokens would show
                compare(whole, *args, causal(n, t, window) & ~gone, d ** -0.5, kind)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("way", WAYS)
def test_a_sequence_without_any_good_page_gives_zeros(kind, way):
    w, q, t, heads = world(way, kind, seed=62)
    o, lse = ask(w, q, t, heads, table=torch.full_like(w.table, w.cache.pages))
    with pytest.raises(bd.BdError) as e:
        bd.poll_status()
    assert e.value.status == 10 and (o == 0).all() and (lse == -np.inf).all()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("power", [-100, 90, 116, 119])
def test_queries_of_any_finite_size_give_what_their_scores_say(way, power):
    """bf16 queries from 2^-100 to about 2^121, the scale making ordinary scores of them."""
    kind = torch.bfloat16
    w, q, t, heads = world(way, kind, seed=71)
    q = bits_of(np.ldexp(values_of(q, kind), power), kind)
    scale = w.d ** -0.5 * 2.0 ** -power
    s = w.seqs[0]
    for cap in (0.0, 20.0):
        got = ask(w, q, t, heads, scale=scale, softcap=cap)
        bd.poll_status()
        compare(got, values_of(q, kind), s.keys(), s.values(), causal(s.length, t), scale, kind, cap)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("first", [True, False])
def test_a_long_flat_tail_beside_a_dominant_token_keeps_its_weight(kind, way, first):
    """One token with a score of about 17 and a value of zero, all others with a score of 0 (2^-24.5 of its weight) and values
    of about 1: the result is the tail's alone."""
    d, heads, kv_heads, n, t = WAYS[way]
    rng = np.random.default_rng(80)
    w = World(1, kv_heads, d, 32, kind, seed=81, max_tokens=n)
    common = rng.choice([-1.0, 1.0], d)
    k, v = np.zeros((n, kv_heads, d)), 1.0 + 0.2 * rng.random((n, kv_heads, d))
    top = 3 if first else n - t - 1
    k[top], v[top] = 17.0 / d ** 0.5 * common, 0.0
    k, v = bits_of(k, kind), bits_of(v, kind)
    w.seqs[0].append(k, v)
    bd.paged_append(w.cache, w.batch([n]), to_device(k, kind), to_device(v, kind))
    q = bits_of(np.broadcast_to(common, (t, heads, d)), kind)
    got = ask(w, q, t, heads)
    bd.poll_status()
    s = w.seqs[0]
    compare(got, values_of(q, kind), s.keys(), s.values(), causal(n, t), d ** -0.5, kind)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -122, -(2.0 ** -122), 2.0 ** -126])
def test_scales_at_the_bottom_of_the_range(way, scale):
    """Queries and keys of about 2^58 each, so that scales below 1e-36 matter; a scale of zero weighs all tokens alike."""
    kind = torch.bfloat16
    d, heads, kv_heads, n, t = WAYS[way]
    rng = np.random.default_rng(90)
    w = World(1, kv_heads, d, 32, kind, seed=91, max_tokens=n)
    k, v = source_rows(rng, n, kv_heads, d, torch.float32)
    k, v = bits_of(np.ldexp(k, 58), kind), bits_of(v, kind)
    w.seqs[0].append(k, v)
    bd.paged_append(w.cache, w.batch([n]), to_device(k, kind), to_device(v, kind))
    q = bits_of(np.ldexp(rng.standard_normal((t, heads, d)), 58), kind)
    s = w.seqs[0]
    for cap in (0.0, 3.0):
        got = ask(w, q, t, heads, scale=scale, softcap=cap)
        bd.poll_status()
        compare(got, values_of(q, kind), s.keys(), s.values(), causal(n, t), scale, kind, cap)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("way", WAYS)
def test_captured_calls_follow_the_numbers_on_the_device(kind, way):
    """A step captured with the bounds of its longest sequence, replayed with other lengths, row counts, pages and queries."""
    d, heads, kv_heads, n, t = WAYS[way]
    w, q0, _, _ = world(way, kind, seed=100)
    s = w.seqs[0]
    keys, values = s.keys(), s.values()
    kv_len, start, table = i32([n]), i32([0, t]), w.table.clone()
    b = bd.PagedBatch(table, w.slots, kv_len, start, t)
    q, out, lse = to_device(q0, kind), torch.empty(t, heads, d, device="cuda"), torch.empty(t, heads, device="cuda")
    workspace = torch.empty(max(256, bd.paged_attention_workspace_size(w.cache, b, t, heads)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.paged_attention(w.cache, b, q, out=out, lse=lse, workspace=workspace)
    order = torch.from_numpy(w.rng.permutation(w.cache.pages)).cuda()           # the same records in other pages
    moved = torch.empty_like(w.cache.pool)
    moved[order] = w.cache.pool
    for length, rows, other in ((n, t, False), (n // 32 * 32, t, True), (n // 64 * 32, max(1, t // 2), True), (32, 1, False), (n, 1, True), (n // 32 * 32, 0, False), (n, t, False)):
        bits = bits_of(w.rng.standard_normal((t, heads, d)), kind)
        q.copy_(to_device(bits, kind))
        kv_len.fill_(length)
        start[1] = rows
        table.copy_(order[w.table.long()].to(torch.int32) if other else w.table)
        pool = w.cache.pool.clone()
        if other:
            w.cache.pool.copy_(moved)
        workspace.fill_(255), out.fill_(-7), lse.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        bd.poll_status()
        w.cache.pool.copy_(pool)
        assert (out[rows:] == -7).all() and (lse[rows:] == -7).all()
        if rows:
            # (kernels and roundings go by the bounds)
            compare((out[:rows].double().cpu().numpy(), lse[:rows].double().cpu().numpy()), values_of(bits, kind)[:rows], keys[:, :length], values_of_prefix(s, length, values),
                    causal(length, rows), d ** -0.5, kind, wide=heads // kv_heads * t > 16)


def values_of_prefix(s, length, values):
    """The stored values of the first `length` tokens: a whole number of chunks, or all."""
    assert length % 32 == 0 or length == s.length
    return values[:, :length]


def test_the_largest_batch():
    """65535 sequences: grids at their limit, unit numbers found by scanning two thousand groups."""
    n, d, heads, kind = 65535, 64, 4, torch.bfloat16
    rng = np.random.default_rng(110)
    cache = bd.PagedKVCache(2 * n, 1, d, n, 32, kind)
    table = torch.randperm(2 * n, device="cuda").to(torch.int32).view(n, 2)
    slots = torch.randperm(n, device="cuda").to(torch.int32)
    length = torch.from_numpy(rng.integers(0, 65, n).astype(np.int32)).cuda()
    start = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    start[1:] = length.cumsum(0)
    total = int(start[-1])
    k, v = (torch.randn(total, 1, d, device="cuda").to(kind) for _ in range(2))
    whole = bd.PagedBatch(table, slots, length, start, 64)
    bd.paged_append(cache, whole, k, v)
    rk, rv = (x.double().cpu().numpy() for x in bd.paged_read(cache, whole, total))
    for t in (1, 5):                                                # few rows; 20 rows: the tensor-core kernel, more tiles than a CTA orders
        q = torch.randn(n * t, heads, d, device="cuda").to(kind)
        lse = torch.empty(n * t, heads, device="cuda")
        o = bd.paged_attention(cache, bd.PagedBatch(table, slots, length, torch.arange(0, n * t + 1, t, dtype=torch.int32, device="cuda"), t), q, dtype=torch.float32, lse=lse)
        bd.poll_status()
        for i in [0, 1, 31, 32, 33, 1023, 1024, 40000, n - 2, n - 1] + [int(x) for x in rng.integers(0, n, 200)]:
            a, m = int(start[i]), int(length[i])
            at = slice(i * t, i * t + t)
            got = o[at].double().cpu().numpy(), lse[at].double().cpu().numpy()
            compare(got, q[at].double().cpu().numpy(), rk[a:a + m].transpose(1, 0, 2), rv[a:a + m].transpose(1, 0, 2), causal(m, t), d ** -0.5, kind) if m else None
            assert m or ((got[0] == 0).all() and (got[1] == -np.inf).all())
        if t == 1:
            workspace = bd.paged_attention_workspace_size(cache, bd.PagedBatch(table, slots, length, start, 1), n, heads)
            assert workspace > 0


def test_queries_that_do_not_fit_are_refused():
    w = World(1, 2, 64, 32, torch.bfloat16, seed=120, max_tokens=64)
    b = w.batch([1], kv_len=[1])
    x = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (x.half(), x.float(), x[:, :3], torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda"), x.cpu(), x[0], x[..., None],
                torch.zeros(1, 64, 4, dtype=torch.bfloat16, device="cuda").transpose(1, 2), None):
        with pytest.raises(ValueError):
            bd.paged_attention(w.cache, b, bad)
    for kw in (dict(out=x[:, :2]), dict(out=x.cpu()), dict(out=x.double()), dict(lse=torch.zeros(1, 2, device="cuda")), dict(lse=torch.zeros(1, 4)), dict(dtype=torch.float64),
               dict(workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            bd.paged_attention(w.cache, b, x, **kw)
    for kw in (dict(window=-1), dict(softcap=-1.0), dict(scale=float("nan")), dict(softcap=float("inf"))):
        with pytest.raises(bd.BdError):
            bd.paged_attention(w.cache, b, x, **kw)
    bd.poll_status()
