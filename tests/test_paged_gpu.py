"""The paged cache on the GPU: append, read back, attention and rotation against the oracle in 64 bits."""
import copy

import numpy as np
import pytest
import torch

import oracle
import paper_2501_01144_b200 as bd
from oracle.paged import attention, norm_rope
from paged_util import World, source_rows, values_of
from paper_2501_01144_b200 import inputs
from util import ORACLE_DTYPE, to_device

pytestmark = pytest.mark.gpu
KINDS = [torch.bfloat16, torch.float16, torch.float32]
HALF_STEP = {k: torch.finfo(k).eps / 2 for k in KINDS}


def i32(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


def rounded(x, kind):
    """fp64 values in the type `kind`, back as fp64."""
    return torch.from_numpy(x).to(kind).double().numpy()


# ---- append and read back -------------------------------------------------------------------------------------------


def check_read(w, back=None):
    new = [min(b, s.length) for b, s in zip(back or w.lengths(), w.seqs)]
    if not sum(new):
        return
    b = w.batch(new)
    k, v = (t.double().cpu().numpy() for t in bd.paged_read(w.cache, b, sum(new)))
    at = 0
    for s, t in zip(w.seqs, new):
        if t:
            wk, wv = (rounded(np.ascontiguousarray(x[:, s.length - t:].transpose(1, 0, 2)), w.kind) for x in (s.keys(), s.values()))
            assert np.array_equal(k[at:at + t], wk), "keys"
            assert np.array_equal(v[at:at + t], wv), "values"
        at += t


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 96])
def test_appends_in_uneven_pieces_read_back_as_the_oracle_says(kind, d, page):
    w = World(4, 2, d, page, kind, seed=d + page, max_tokens=300)
    for new in ([1, 31, 32, 0], [1, 1, 33, 0], [30, 0, 1, 5], [40, 64, 63, 27], [1, 1, 1, 1], [3, 100, 31, 64]):
        w.step(new)
        check_read(w)
        check_read(w, [1, 7, 33, 500])
    bd.poll_status()


def test_stored_records_have_the_documented_layout():
    """Codes, ids and scales of the pool, decoded byte by byte from the header's description, against the oracle's bits."""
    d, nb, n, kind = 128, 4, 75, torch.bfloat16
    w = World(1, 2, d, 64, kind, seed=5, max_tokens=n)
    w.step([20])
    w.step([55])
    pool, table = w.cache.pool.cpu().numpy(), w.table.cpu().numpy()[0]
    nibble = [0, 2, 1, 3, 4, 6, 5, 7]
    for h in range(2):
        ref = w.seqs[0].heads[h]
        kc, ki, ks = ref.keys()
        vc, vi, vs = ref.values_quantised()

        def block(rec, key, b, r):
            g, j = r % 8, r // 8
            words = rec[(0 if key else 16 * d):][: 16 * d].view(np.uint32)
            codes = [(int(words[((8 * b + g) * 4 + t) * 4 + j]) >> (4 * nibble[e])) & 15 for t in range(4) for e in range(8)]
            e = (4 * g + j) * nb + b
            ids = rec[(34 * d if key else 34 * d + d // 2):]
            return codes, (int(ids[e // 2]) >> (4 * (e % 2))) & 15, int(rec[(32 * d if key else 33 * d) + e])

        def want(c, i, s, row, blk):
            by = c[row, 16 * blk:16 * blk + 16]
            return [int(x) for y in by for x in (y & 15, y >> 4)], int(i[row, blk]), int(s[row, blk])

        for tok in range(n):
            c, k = tok // 32, tok % 32
            rec = pool[table[c // 2], h, c % 2]
            for b in range(nb):
                assert block(rec, True, b, 8 * (k // 2 % 4) + 2 * (k // 8) + k % 2) == want(kc, ki, ks, tok, b)
        for c in range(n // 32):
            rec = pool[table[c // 2], h, c % 2]
            for ch in range(d):
                assert block(rec, False, ch // 32, ch % 32) == want(vc, vi, vs, ch, c)


def test_nothing_but_the_step_changes():
    """Other pages, other slots, other tokens' bytes of the same chunk and rows behind the last sequence keep their bytes."""
    w = World(2, 2, 64, 32, torch.float16, seed=6, max_tokens=100)
    w.step([37, 5])
    pool, tail = w.cache.pool.clone(), w.cache.tail.clone()
    rows = [to_device(x, torch.float16) for x in source_rows(w.rng, 6, 2, 64, torch.float16)]
    b = bd.PagedBatch(w.table, w.slots, i32([39, 5]), i32([1, 3, 3]), 4)          # two tokens for sequence 0 from rows 1, 2 of 6
    bd.paged_append(w.cache, b, *rows)
    touched = (w.cache.pool != pool).nonzero()
    assert len(touched) and (touched[:, 0] == w.table[0, 1]).all()                # page of tokens 32 .. 63 of sequence 0
    per = (w.cache.pool != pool)[w.table[0, 1].item(), 0, 0]
    assert per[16 * 64:32 * 64].sum() == 0 and per[33 * 64:34 * 64].sum() == 0    # no value bytes: the chunk is unfinished
    assert per[:16 * 64].sum() <= 2 * 32 and per[32 * 64:33 * 64].sum() <= 2 * 2
    same = w.cache.tail.view(torch.int16) == tail.view(torch.int16)
    same[w.slots[0].long(), :, 37:39] = True
    assert same.all()
    # read back: rows in front of and behind the sequences' own stay as they were
    k, v = (torch.full((7, 2, 64), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    bd.paged_read(w.cache, bd.PagedBatch(w.table, w.slots, i32([39, 5]), i32([1, 3, 5]), 4), out_k=k, out_v=v)
    for x in (k, v):
        assert (x[0] == 3).all() and (x[5:] == 3).all() and not (x[1:5] == 3).all(-1).any()
    bd.poll_status()


@pytest.mark.parametrize("old,t", [(0, 32), (31, 1), (31, 32), (45, 20), (64, 9), (63, 2)])
def test_a_step_can_be_repeated_and_taken_back(old, t):
    w = World(1, 1, 64, 64, torch.bfloat16, seed=7 + old, max_tokens=200)
    if old:
        w.step([old])
    b, k, v = w.step([t])
    state = [x.clone() for x in bd.paged_read(w.cache, w.batch([old + t]), old + t)]
    bd.paged_append(w.cache, b, to_device(k, w.kind), to_device(v, w.kind))     # again
    assert all(torch.equal(x, y) for x, y in zip(state, bd.paged_read(w.cache, w.batch([old + t]), old + t)))
    # other tokens were drafted behind these and are taken back: up to 32 of them
    dk, dv = (to_device(x, w.kind) for x in source_rows(w.rng, 32, 1, 64, w.kind))
    bd.paged_append(w.cache, bd.PagedBatch(w.table, w.slots, i32([old + t + 32]), i32([0, 32]), 32), dk, dv)
    assert all(torch.equal(x, y) for x, y in zip(state, bd.paged_read(w.cache, w.batch([old + t]), old + t)))
    w.step([40])
    check_read(w)


def test_strided_sources_and_destinations():
    """Keys and values as slices of one projection's rows, results as slices of one buffer, and heads outermost."""
    t, hk, d, kind = 70, 2, 128, torch.bfloat16
    w = World(1, hk, d, 64, kind, seed=8, max_tokens=100)
    k, v = source_rows(w.rng, t, hk, d, kind)
    w.seqs[0].append(k, v)
    buf = torch.zeros(t, 5 * hk * d, dtype=kind, device="cuda")
    ks, vs = (buf[:, i * hk * d:(i + 1) * hk * d].view(t, hk, d) for i in (1, 3))
    ks.copy_(to_device(k, kind)), vs.copy_(to_device(v, kind))
    bd.paged_append(w.cache, w.batch([t]), ks, vs)
    check_read(w)
    got = torch.zeros(2, hk, t, d, dtype=kind, device="cuda").transpose(1, 2)     # [2][t, hk, d] with the heads outermost in memory
    bd.paged_read(w.cache, w.batch([t]), out_k=got[0], out_v=got[1])
    assert np.array_equal(got[0].double().cpu().numpy(), w.seqs[0].keys().transpose(1, 0, 2))
    assert np.array_equal(got[1].double().cpu().numpy(), w.seqs[0].values().transpose(1, 0, 2))


def test_nonfinite_keys_are_reported():
    w = World(1, 1, 64, 32, torch.bfloat16, seed=9, max_tokens=64)
    k, v = (torch.ones(3, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[1, 0, 7] = float("inf")
    bd.paged_append(w.cache, bd.PagedBatch(w.table, w.slots, i32([3]), i32([0, 3]), 3), k, v)
    with pytest.raises(bd.BdError) as e:
        bd.poll_status()
    assert e.value.status == 6
    bd.poll_status()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_nonfinite_values_are_reported_with_the_step_that_brings_them(kind, d, value):
    """Also while their chunk is unfinished and no quantizer has met them; the largest finite value is none of them."""
    w = World(2, 2, d, 32, kind, seed=48, max_tokens=64)
    w.step([30, 3])
    for row, head, ch in ((0, 0, 0), (0, 1, d - 1), (1, 0, 7), (2, 1, 33)):
        k, v = (torch.zeros(3, 2, d, dtype=kind, device="cuda") for _ in range(2))
        v[:] = torch.finfo(kind).max
        b = bd.PagedBatch(w.table, w.slots, i32([31, 5]), i32([0, 1, 3]), 2)
        bd.paged_append(w.cache, b, k, v)
        bd.poll_status()
        v[row, head, ch] = value
        bd.paged_append(w.cache, b, k, v)
        with pytest.raises(bd.BdError) as e:
            bd.poll_status()
        assert e.value.status == 6
        bd.poll_status()


# ---- attention ------------------------------------------------------------------------------------------------------


def queries(rng, rows, heads, d, kind, spread=1.0):
    q = (rng.standard_normal((rows, heads, d)) * spread).astype(np.float32)
    bits = inputs.to_bf16_bits(q) if kind == torch.bfloat16 else inputs.to_f16_bits(q)
    return bits, values_of(bits, kind)


def check_attention(w, new, heads, out_dtype=torch.float32, softcap=0.0, window=0, scale=None, spread=1.0):
    w.step(new)
    # probabilities meet the values in fp16; calls of more than 16 rows per KV head round them to the cache's type
    p_half_step = HALF_STEP[w.kind] if heads // w.kv_heads * max(new) > 16 else HALF_STEP[torch.float16]
    b = w.batch(new)
    rows = sum(new)
    bits, q = queries(w.rng, rows, heads, w.d, w.kind, spread)
    scale = w.d ** -0.5 if scale is None else scale
    lse = torch.full((rows, heads), 7.0, device="cuda")
    o = bd.paged_attention(w.cache, b, to_device(bits, w.kind), scale=scale, softcap=softcap, window=window, dtype=out_dtype, lse=lse)
    bd.poll_status()
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    at = 0
    for s, t in zip(w.seqs, new):
        if t:
            ro, rl, pv, qk, vv = attention(q[at:at + t], s.keys(), s.values(), scale, softcap, window)
            # scores: exact products, fp32 sums over at most 128 of them, a few fp32 operations after (and the exponential's argument in units of log2 e)
            ds = (128 + 8) * 2.0 ** -24 * scale * qk + 2.0 ** -20 * (softcap or 0.0) + 2.0 ** -22 * (np.abs(np.where(np.isinf(rl), 0, rl))[..., None] + 1)
            # probabilities: half a step of their 16-bit form, 2^-22 of the exponential, an absolute 2^-25 below fp16's normal range; sums over the tokens in fp32
            rel = p_half_step + 2 * ds + 2.0 ** -21 + s.length * 2.0 ** -24
            # (calls of more than 16 rows on fp16 caches hold the values in fp16: half a step of its subnormals, 2^-25, each)
            bound = rel * pv + 2.0 ** -25 * vv + 2.0 ** -25 * (w.kind == torch.float16) + HALF_STEP[out_dtype] * np.abs(ro) + 2.0 ** -24 * (out_dtype == torch.float16)
            err = np.abs(o[at:at + t] - ro)
            assert (err <= bound).all(), f"max error / bound {np.nanmax(err / np.maximum(bound, 1e-300))}, t {t} of {s.length}"
            seen = np.isfinite(rl)
            assert (np.isinf(lse[at:at + t]) == ~seen).all() and (o[at:at + t][~seen] == 0).all()
            assert (np.abs(np.where(seen, lse[at:at + t], 0) - np.where(seen, rl, 0)) <= 2 * ds.max(-1) + 2.0 ** -20 + s.length * 2.0 ** -24).all()
        at += t


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,heads,kv_heads", [(128, 8, 2), (64, 2, 2), (128, 14, 2), (64, 16, 1)])
def test_single_tokens(kind, d, heads, kv_heads):
    w = World(5, kv_heads, d, 64, kind, seed=heads, max_tokens=700)
    w.step([0, 30, 31, 256, 640])
    check_attention(w, [1, 1, 1, 1, 1], heads)                      # lengths 1, 31, 32, 257, 641
    check_attention(w, [1, 0, 1, 1, 1], heads, out_dtype=kind)      # one of them has nothing to do


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,heads,kv_heads,page", [(128, 8, 2, 32), (64, 6, 2, 96), (128, 3, 3, 64)])
@pytest.mark.parametrize("softcap,window", [(0.0, 0), (20.0, 0), (0.0, 50), (5.0, 1), (0.0, 33)])
def test_a_few_tokens_with_caps_and_windows(kind, d, heads, kv_heads, page, softcap, window):
    w = World(4, kv_heads, d, page, kind, seed=page, max_tokens=400)
    w.step([0, 17, 95, 300])
    check_attention(w, [3, 5, 1, 2], heads, softcap=softcap, window=window, spread=2.0)
    check_attention(w, [4, 1, 33, 2], heads, out_dtype=kind, softcap=softcap, window=window)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_of_prompts(kind, d):
    w = World(3, 2, d, 64, kind, seed=20 + d, max_tokens=520)
    check_attention(w, [33, 1, 200], 4)
    check_attention(w, [130, 64, 257], 4, out_dtype=kind)
    check_attention(w, [129, 0, 31], 4, window=100, softcap=10.0)


def test_long_context_is_split_and_joined():
    w = World(1, 1, 128, 128, torch.bfloat16, seed=30, max_tokens=9000)
    w.step([8920])
    check_attention(w, [1], 4)
    check_attention(w, [2], 1, window=4000)
    check_attention(w, [5], 4)                                      # 20 rows: the tensor-core kernel, its tokens shared by CTAs
    check_attention(w, [33], 4, window=3000, softcap=15.0)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("softcap,window", [(0.0, 0), (12.0, 6200)])
def test_many_rows_over_a_long_context(kind, softcap, window):
    """Tiles expanded in front (about 4096 rows and 6144 tokens or more, head_dim 128), with an unfinished chunk."""
    w = World(2, 1, 128, 64, kind, seed=36, max_tokens=7000)
    w.step([6390, 3])
    # the images of two sequences' 55 tiles, 128 keys and values of 256 bytes each
    assert bd.paged_attention_workspace_size(w.cache, w.batch([512, 1]), 513, 8) >= 2 * 55 * 2 * 128 * 256
    check_attention(w, [512, 40], 8, softcap=softcap, window=window)
    # a page number outside the pool: its tokens are not seen, by this kernel or the one for few rows
    bits, _ = queries(w.rng, 513, 8, 128, kind)
    q, table = to_device(bits, kind), w.table.clone()
    table[0, 20] = -7
    many = bd.paged_attention(w.cache, bd.PagedBatch(table, w.slots, i32([6902, 43]), i32([0, 512, 513]), 512), q, softcap=softcap, window=window, dtype=torch.float32)
    few = bd.paged_attention(w.cache, bd.PagedBatch(table, w.slots, i32([6902, 43]), i32([0, 2, 3]), 2), torch.cat([q[510:512], q[512:]]), softcap=softcap, window=window, dtype=torch.float32)
    with pytest.raises(bd.BdError):
        bd.poll_status()
    assert (many[510:] - few).abs().max() <= 2 * (HALF_STEP[kind] + 2.0 ** -11) * w.cache.head_dim ** 0.5 * 4 and torch.isfinite(many).all()


@pytest.mark.parametrize("heads,most", [(4, 1), (8, 4), (16, 4)])
def test_many_ragged_sequences_share_the_warps(heads, most):
    """More sequences than a scan's 32 lanes, lengths from nothing to two pages of chunks: runs that cross heads and sequences."""
    n = 75
    w = World(n, 2, 64, 96, torch.bfloat16, seed=37, max_tokens=1500)
    old = [0 if i % 7 == 3 else 1 + (i * 37) % 120 for i in range(n)]
    old[5], old[60], old[74] = 1400, 1111, 900
    w.step(old)
    new = [0 if i % 5 == 1 else 1 + i % most for i in range(n)]
    if most * heads // 2 <= 16:                                     # (more rows: the tensor-core kernel, no need to share)
        assert bd.paged_attention_workspace_size(w.cache, w.batch(new), sum(new), heads) > 0
    check_attention(w, new, heads)
    check_attention(w, new[::-1], heads, window=500)


def test_more_row_tiles_than_a_cta_orders():
    n = 530
    w = World(n, 1, 64, 32, torch.bfloat16, seed=38, max_tokens=64)
    w.step([i % 9 for i in range(n)])
    check_attention(w, [5 if i % 11 == 0 else i % 3 for i in range(n)], 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [2.0 ** -120, 2.0 ** -20, 2.0 ** -11, 2.0 ** 8])
def test_magnitudes_at_the_ends_of_the_types(kind, scale):
    if kind == torch.float16 and scale < 2.0 ** -20:
        pytest.skip("below fp16's range")
    w = World(1, 2, 128, 32, kind, seed=39, max_tokens=128)
    k, v = source_rows(w.rng, 75, 2, 128, torch.float32)
    conv = {torch.float32: lambda x: x, torch.bfloat16: inputs.to_bf16_bits, torch.float16: inputs.to_f16_bits}[kind]
    k, v = conv((k * scale).astype(np.float32)), conv((v * scale).astype(np.float32))
    w.seqs[0].append(k, v)
    bd.paged_append(w.cache, w.batch([75]), to_device(k, kind), to_device(v, kind))
    check_read(w)
    if kind != torch.float32 and scale > 2.0 ** -100:
        w.kind = kind
        check = dict(scale=128 ** -0.5 / scale)
        check_attention(w, [1], 4, **check)
        check_attention(w, [40], 4, **check)


def test_a_pool_beyond_32_bits():
    """Pages whose records lie more than 2^32 bytes into the pool."""
    hk, d, page = 8, 128, 64
    pages = (1 << 32) // (hk * 2 * 35 * d) + 60
    w = World.__new__(World)
    w.rng, w.n, w.kv_heads, w.d, w.page, w.kind = np.random.default_rng(41), 1, hk, d, page, torch.bfloat16
    w.table = i32([[pages - 1 - 3 * i for i in range(12)]])
    w.slots = i32([2])
    w.cache = bd.PagedKVCache(pages, hk, d, 3, page, w.kind)
    from oracle.paged import Sequence
    w.seqs = [Sequence(hk, d, ORACLE_DTYPE[w.kind])]
    assert int(w.table[0, 11]) * hk * 2 * 35 * d > 1 << 32
    w.step([300])
    check_read(w)
    check_attention(w, [1], 8)
    check_attention(w, [30], 8)


def test_another_formatbook_reaches_the_paged_kernels():
    book = oracle.formatbook().copy()
    book[0, 6], book[1, 6] = 13, 9                                  # another member of the first pair
    try:
        bd.set_formatbook(book)
        oracle.set_formatbook(book)
        w = World(1, 1, 128, 32, torch.bfloat16, seed=43, max_tokens=200)
        w.step([77])
        check_read(w)
        check_attention(w, [1], 4)
        check_attention(w, [60], 4)
    finally:
        bd.set_formatbook(None)
        oracle.set_formatbook(None)


def test_sharp_rows_and_tiny_and_huge_queries():
    w = World(2, 1, 128, 64, torch.bfloat16, seed=31, max_tokens=300)
    w.step([200, 250])
    for spread in (30.0, 1e-3, 1e-30, 1e4):
        check_attention(w, [1, 2], 4, spread=spread, scale=1.0 / (spread * 11.0) if spread > 100 else None)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,heads,old,new,window", [
    (128, 4, 300, 2, 40), (64, 16, 1900, 1, 1100),                  # few rows: a CTA per head, runs
    (64, 4, 690, 40, 100), (128, 2, 2900, 33, 700),                 # more rows: alone, shared by CTAs
    (128, 8, 6800, 512, 6200)])                                     # tiles expanded in front
def test_pages_in_front_of_the_window_may_be_gone(kind, d, heads, old, new, window):
    n = old + new
    w = World(1, 1, d, 32, kind, seed=window, max_tokens=n)
    k, v = (to_device(x, kind) for x in source_rows(w.rng, n, 1, d, kind))
    bd.paged_append(w.cache, bd.PagedBatch(w.table, w.slots, i32([n]), i32([0, n]), n), k, v)
    q = to_device(queries(w.rng, new, heads, d, kind)[0], kind)
    want, lse = (torch.empty(new, heads, d, device="cuda"), torch.empty(new, heads, device="cuda"))
    bd.paged_attention(w.cache, bd.PagedBatch(w.table, w.slots, i32([n]), i32([0, new]), new), q, window=window, out=want, lse=lse)
    gone = (old - window + 1) // 32
    assert gone > 0 and torch.isfinite(want).all()
    junk = next(p for p in range(w.cache.pages) if p not in w.table[0].tolist())      # a page that nobody wrote
    for number in (-1, w.cache.pages, junk):
        table = w.table.clone()
        table[0, :gone] = number
        b = bd.PagedBatch(table, w.slots, i32([n]), i32([0, new]), new)
        got_lse = torch.empty_like(lse)
        got = bd.paged_attention(w.cache, b, q, window=window, dtype=torch.float32, lse=got_lse)
        bd.poll_status()
        assert torch.equal(got, want) and torch.equal(got_lse, lse)


def test_rows_that_see_nothing_give_zeros():
    w = World(2, 2, 128, 32, torch.bfloat16, seed=32, max_tokens=64)
    w.step([2, 40])
    b = w.batch([5, 1])                                             # sequence 0: five rows, two tokens
    q = to_device(queries(w.rng, 6, 4, 128, w.kind)[0], w.kind)
    lse = torch.zeros(6, 4, device="cuda")
    o = bd.paged_attention(w.cache, b, q, lse=lse)
    assert (o[:3] == 0).all() and torch.isinf(lse[:3]).all() and not (o[3:] == 0).all(-1).any() and torch.isfinite(lse[3:]).all()
    b = w.batch([5, 1], kv_len=[0, 0])                              # empty caches
    assert (bd.paged_attention(w.cache, b, q) == 0).all()
    bd.poll_status()


def test_padding_rows_stay_and_results_repeat():
    w = World(3, 2, 128, 64, torch.bfloat16, seed=33, max_tokens=500)
    w.step([100, 450, 7])
    q = to_device(queries(w.rng, 9, 8, 128, w.kind)[0], w.kind)
    out = torch.full((9, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((9, 8), 5.0, device="cuda")
    b = bd.PagedBatch(w.table, w.slots, i32(w.lengths()), i32([1, 3, 3, 6]), 4)
    bd.paged_attention(w.cache, b, q, out=out, lse=lse)
    for x in (out, lse):
        assert (x[0] == 5).all() and (x[6:] == 5).all() and not (x[1:6] == 5).any(-1).all()
    again = bd.paged_attention(w.cache, b, q)
    assert torch.equal(out[1:6], again[1:6])
    # a sequence alone gives what it gives in the batch when the launch is cut alike
    alone = bd.paged_attention(w.cache, bd.PagedBatch(w.table[2:], w.slots[2:], i32(w.lengths()[2:]), i32([0, 3]), 4), q[3:6])
    assert (alone.float() - out[3:6].float()).abs().max() <= 2.0 ** -7 * out[3:6].float().abs().max()


def test_pages_and_slots_out_of_range_are_reported_and_not_followed():
    w = World(2, 1, 64, 32, torch.bfloat16, seed=34, max_tokens=128)
    w.step([100, 100])
    q = to_device(queries(w.rng, 2, 2, 64, w.kind)[0], w.kind)
    good = bd.paged_attention(w.cache, w.batch([1, 1]), q)

    def reported():
        with pytest.raises(bd.BdError) as e:
            bd.poll_status()
        assert e.value.status == 10
        bd.poll_status()

    for bad in (-1, w.cache.pages, 2 ** 31 - 1):
        table = w.table.clone()
        table[0, 1] = bad
        b = bd.PagedBatch(table, w.slots, i32([100, 100]), i32([0, 1, 2]), 1)
        o = bd.paged_attention(w.cache, b, q)
        assert torch.equal(o[1], good[1]) and torch.isfinite(o).all()
        reported()
        k, v = bd.paged_read(w.cache, bd.PagedBatch(table, w.slots, i32([100, 100]), i32([0, 100, 101]), 100), 101)
        assert (k[32:64] == 0).all() and (v[32:64] == 0).all() and (k[64:100] != 0).any()
        reported()
        before = w.cache.pool.clone()
        x = torch.ones(32, 1, 64, dtype=torch.bfloat16, device="cuda")
        bd.paged_append(w.cache, bd.PagedBatch(table, w.slots, i32([64, 100]), i32([0, 32, 32]), 32), x, x)
        assert torch.equal(before, w.cache.pool)
        reported()
    for slot in (-1, w.cache.slots):
        before, tail = w.cache.pool.clone(), w.cache.tail.view(torch.int16).clone()
        b = bd.PagedBatch(w.table, i32([slot, w.slots[1].item()]), i32([101, 100]), i32([0, 1, 1]), 1)
        x = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
        bd.paged_append(w.cache, b, x, x)
        assert torch.equal(before, w.cache.pool) and torch.equal(tail, w.cache.tail.view(torch.int16))
        reported()
        assert torch.isfinite(bd.paged_attention(w.cache, bd.PagedBatch(w.table, i32([slot, w.slots[1].item()]), i32([100, 100]), i32([0, 1, 2]), 1), q)).all()
        reported()
    for kv, start in (([-5, 100], [0, 1, 2]), ([100, 129], [0, 1, 2]), ([100, 100], [0, -1, 1]), ([100, 100], [0, 1, 9])):
        out = torch.full((2, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        bd.paged_attention(w.cache, bd.PagedBatch(w.table, w.slots, i32(kv), i32(start), 2), q, out=out)
        reported()


def test_sequences_without_rows_need_no_slot_and_no_pages():
    """A padded batch: entries without rows carry -1 for slot and pages."""
    w = World(2, 2, 64, 32, torch.bfloat16, seed=36, max_tokens=64)
    w.step([20, 13])
    table, slots = torch.cat([w.table, torch.full_like(w.table, -1)]), torch.cat([w.slots, torch.full_like(w.slots, -1)])
    rows = [source_rows(w.rng, 1, 2, 64, w.kind) for _ in range(2)]
    for s, (k, v) in zip(w.seqs, rows):
        s.append(k, v)
    b = bd.PagedBatch(table, slots, i32([21, 14, 0, 0]), i32([0, 1, 2, 2, 2]), 1)
    bd.paged_append(w.cache, b, *(to_device(np.concatenate([r[j] for r in rows]), w.kind) for j in (0, 1)))
    bd.paged_read(w.cache, b, 2)
    bd.paged_attention(w.cache, b, to_device(queries(w.rng, 2, 4, 64, w.kind)[0], w.kind))
    bd.poll_status()
    check_read(w)


def test_binding_refuses_what_does_not_fit():
    w = World(1, 2, 64, 32, torch.bfloat16, seed=35, max_tokens=64)
    b = w.batch([1], kv_len=[1])
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (x.half(), x[:, :1], torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda"), x.cpu(), x[0], torch.zeros(1, 64, 2, dtype=torch.bfloat16, device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            bd.paged_append(w.cache, b, bad, x)
        with pytest.raises(ValueError):
            bd.paged_attention(w.cache, b, bad) if bad.dim() != 3 or bad.shape[1:] != (2, 64) or bad.dtype != x.dtype or not bad.is_cuda or bad.stride(2) != 1 else bd.paged_append(w.cache, b, x, bad)
    with pytest.raises(ValueError):
        bd.PagedBatch(w.table.long(), w.slots, i32([1]), i32([0, 1]), 1)
    with pytest.raises(ValueError):
        bd.PagedBatch(w.table, w.slots, i32([1]), i32([0, 1, 2]), 1)
    with pytest.raises(ValueError):
        bd.paged_append(w.cache, bd.PagedBatch(w.table, w.slots, i32([1]), i32([0, 1]), 1, max_kv=10 ** 6), x, x)
    with pytest.raises(ValueError):
        bd.PagedKVCache.from_buffers(w.cache.pool, w.cache.tail, 64)
    with pytest.raises(ValueError):
        bd.paged_attention(w.cache, b, torch.zeros(1, 3, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(bd.BdError) as e:
        bd.paged_attention(w.cache, b, x, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"), dtype=torch.float16)
    assert e.value.status == 4
    bd.poll_status()


def test_members_of_caches_and_batches_are_fixed():
    """Their descriptors hold the tensors' addresses: another tensor in a member's place would not be seen."""
    w = World(1, 2, 64, 32, torch.bfloat16, seed=37, max_tokens=64)
    b = w.batch([1], kv_len=[1])
    for obj, name in ((w.cache, "pool"), (w.cache, "tail"), (w.cache, "page_tokens"), (b, "kv_len"), (b, "page_table"), (b, "max_kv")):
        with pytest.raises(AttributeError):
            setattr(obj, name, getattr(obj, name))
        with pytest.raises(AttributeError):
            delattr(obj, name)
    b.kv_len.fill_(0)                                               # contents may change
    assert (bd.paged_attention(w.cache, b, torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda")) == 0).all()


def test_a_forked_cache_has_buffers_of_its_own():
    """deepcopy: what is appended to the copy shows in the copy alone, and it outlives the original."""
    w = World(1, 2, 64, 32, torch.bfloat16, seed=47, max_tokens=96)
    w.step([40])
    fork, batch = copy.deepcopy((w.cache, w.batch([45], kv_len=[45])))
    before = [x.clone() for x in bd.paged_read(w.cache, w.batch([40]), 40)]
    pool, tail = w.cache.pool.clone(), w.cache.tail.view(torch.int16).clone()
    k, v = source_rows(w.rng, 5, 2, 64, w.kind)
    bd.paged_append(fork, bd.PagedBatch(w.table, w.slots, i32([45]), i32([0, 5]), 5), to_device(k, w.kind), to_device(v, w.kind))
    assert torch.equal(pool, w.cache.pool) and torch.equal(tail, w.cache.tail.view(torch.int16))
    w.seqs[0].append(k, v)
    w.cache.pool.fill_(255), w.cache.tail.view(torch.int16).fill_(-1), w.table.fill_(-1)
    w.cache = fork
    got = [x.clone() for x in bd.paged_read(fork, batch, 45)]
    assert np.array_equal(got[0].double().cpu().numpy(), w.seqs[0].keys().transpose(1, 0, 2)) and torch.equal(got[0][:40], before[0])
    assert np.array_equal(got[1].double().cpu().numpy(), w.seqs[0].values().transpose(1, 0, 2))
    bd.poll_status()


# ---- rotation -------------------------------------------------------------------------------------------------------


def cos_sin(positions, rot):
    ang = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 32), (64, 64), (64, 16), (128, 80)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,kv_heads,norm", [(1, 4, 1, (True, True)), (37, 7, 3, (True, False)), (5, 32, 8, (False, False)), (3, 1, 0, (True, False))])
def test_rotation_against_the_oracle(kind, d, rot, interleaved, rows, heads, kv_heads, norm):
    rng = np.random.default_rng(d + rot + rows)
    conv = {torch.float32: lambda x: x, torch.bfloat16: inputs.to_bf16_bits, torch.float16: inputs.to_f16_bits}[kind]
    mk = lambda *s: conv((rng.standard_normal(s) * 3).astype(np.float32))  # noqa: E731
    q, k, wq, wk = mk(rows, heads, d), mk(rows, max(kv_heads, 1), d), mk(d), mk(d)
    tab, pos = cos_sin(5000, rot), rng.integers(0, 5000, rows)
    dev = [to_device(x, kind) for x in (q, k, wq, wk)]
    gq, gk = bd.qk_norm_rope(dev[0], dev[1] if kv_heads else None, i32(pos), torch.from_numpy(tab).cuda(), dev[2] if norm[0] else None, dev[3] if norm[1] else None, eps=1e-5,
                             interleaved=interleaved)
    bd.poll_status()
    for got, x, w, use in ((gq, q, wq, norm[0]), (gk, k, wk, norm[1])):
        if got is None:
            continue
        ref = norm_rope(values_of(x, kind), values_of(w, kind) if use else None, tab.astype(np.float64), pos, 1e-5, interleaved)
        size = norm_rope(np.abs(values_of(x, kind)), np.abs(values_of(w, kind)) if use else None, np.concatenate([np.abs(tab[:, :rot // 2]), -np.abs(tab[:, rot // 2:])], 1).astype(np.float64), pos, 1e-5, interleaved)
        # fp32 throughout: the mean (8 sums per lane, 4 levels), reciprocal root (2 ulp), three products, one sum: under 32 * 2^-24 of the terms' sizes; one rounding
        size = np.abs(norm_rope(np.abs(values_of(x, kind)), np.abs(values_of(w, kind)) if use else None, np.abs(tab).astype(np.float64), pos, 1e-5, interleaved)) + np.abs(size)
        bound = 32 * 2.0 ** -24 * size + HALF_STEP[kind] * np.abs(ref) + (2.0 ** -24 if kind == torch.float16 else 0.0)
        assert (np.abs(got.double().cpu().numpy() - ref) <= bound).all()


def test_rotation_in_place_on_slices_and_bad_positions():
    rows, h, hk, d = 6, 4, 2, 128
    rng = np.random.default_rng(1)
    bits = inputs.to_bf16_bits(rng.standard_normal((rows, (h + 2 * hk) * d)).astype(np.float32))
    qkv = to_device(bits, torch.bfloat16)
    tab = torch.from_numpy(cos_sin(100, d)).cuda()
    pos = i32([0, 5, 99, 100, -1, 7])
    q, k = qkv[:, :h * d].view(rows, h, d), qkv[:, h * d:(h + hk) * d].view(rows, hk, d)
    want_q, want_k = bd.qk_norm_rope(q, k, i32([0, 5, 99, 0, 0, 7]), tab)
    before = qkv.clone()
    bd.qk_norm_rope(q, k, pos, tab, out_q=q, out_k=k)
    ok = [0, 1, 2, 5]
    assert torch.equal(q[ok], want_q[ok]) and torch.equal(k[ok], want_k[ok])
    assert torch.equal(qkv[3:5], before[3:5]) and torch.equal(qkv[:, (h + hk) * d:], before[:, (h + hk) * d:])
    with pytest.raises(bd.BdError) as e:
        bd.poll_status()
    assert e.value.status == 10
    e, _ = bd.qk_norm_rope(q[:0], None, pos[:0], tab)
    assert e.shape == (0, h, d)


# ---- the operators together -----------------------------------------------------------------------------------------


def test_a_decode_loop_captured_in_a_graph_and_replayed():
    """Projection, rotation, append, attention and output projection of a layer for three sequences; the step captured
    once and replayed while lengths grow, against the same calls made one by one and against the oracle."""
    n, h, hk, d, hidden, kind = 3, 4, 2, 64, 256, torch.bfloat16
    rng = np.random.default_rng(40)
    wqkv, wo = (bd.quantize_weights(torch.from_numpy((rng.standard_normal(s) * 0.06).astype(np.float32)).cuda(), bd.SELECT_TWO_STAGE) for s in (((h + 2 * hk) * d, hidden), (hidden, h * d)))
    tab = torch.from_numpy(cos_sin(300, d)).cuda()
    weight = torch.ones(d, dtype=kind, device="cuda")

    def world():
        w = World(n, hk, d, 32, kind, seed=41, max_tokens=160)
        w.step([20, 61, 1])
        return w

    def step(w, x, kv_len, starts, ws, out):
        qkv = bd.linear(x, wqkv, workspace=ws[0], out=out[0])
        q, k, v = (t.view(n, -1, d) for t in qkv.split([h * d, hk * d, hk * d], 1))
        bd.qk_norm_rope(q, k, kv_len - 1, tab, weight, weight, out_q=q, out_k=k)
        b = bd.PagedBatch(w.table, w.slots, kv_len, starts, 1)
        bd.paged_append(w.cache, b, k, v)
        bd.paged_attention(w.cache, b, q, out=out[1], workspace=ws[1])
        return bd.linear(out[1].view(n, -1), wo, workspace=ws[2], out=out[2])

    starts = i32([0, 1, 2, 3])
    mk_ws = lambda: [torch.empty(1 << 22, dtype=torch.uint8, device="cuda") for _ in range(3)]  # noqa: E731
    mk_out = lambda: [torch.empty(n, s, dtype=kind, device="cuda") for s in ((h + 2 * hk) * d,)] + [torch.empty(n, h, d, dtype=kind, device="cuda"), torch.empty(n, hidden, dtype=kind, device="cuda")]  # noqa: E731
    xs = [to_device(inputs.to_bf16_bits(rng.standard_normal((n, hidden)).astype(np.float32)), kind) for _ in range(40)]
    lens = torch.tensor([20, 61, 1], dtype=torch.int32, device="cuda")
    eager_w, eager, kv = world(), [], lens.clone()
    ws, out = mk_ws(), mk_out()
    for x in xs:
        kv += 1
        eager.append(step(eager_w, x, kv, starts, ws, out).clone())
    graph_w, x0, kv2 = world(), xs[0].clone(), lens.clone()
    ws2, out2 = mk_ws(), mk_out()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                   # a first call outside the capture; its step is repeated by the first replay
        kv2 += 1
        step(graph_w, x0, kv2, starts, ws2, out2)
        kv2 -= 1
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv2 += 1
        step(graph_w, x0, kv2, starts, ws2, out2)
    for i, x in enumerate(xs):
        x0.copy_(x)
        graph.replay()
        assert torch.equal(out2[2], eager[i]), f"step {i}"
    bd.poll_status()
    # the last step's attention against the oracle, from the cache as it stands
    new = [1, 1, 1]
    total = (lens + 40).tolist()
    k, v = (t.double().cpu().numpy() for t in bd.paged_read(graph_w.cache, graph_w.batch(total, total), sum(total)))
    q = out2[0][:, :h * d].view(n, h, d).double().cpu().numpy()
    at = 0
    for i, m in enumerate(total):
        ro, _, pv, _, vv = attention(q[i:i + 1], k[at:at + m].transpose(1, 0, 2), v[at:at + m].transpose(1, 0, 2), d ** -0.5)
        err = np.abs(out2[1][i].double().cpu().numpy() - ro[0])
        assert (err <= (2.0 ** -11 + 2.0 ** -13) * pv[0] + 2.0 ** -8 * np.abs(ro[0]) + 2.0 ** -25 * vv[0]).all()
        at += m


def test_two_captured_graphs_with_workspaces_of_their_own_and_another_stream():
    w = World(2, 1, 128, 64, torch.bfloat16, seed=42, max_tokens=2000)
    w.step([1900, 700])
    b = w.batch([1, 1])
    qs = [to_device(queries(w.rng, 2, 4, 128, w.kind)[0], w.kind) for _ in range(2)]
    want = [bd.paged_attention(w.cache, b, q) for q in qs]
    assert bd.paged_attention_workspace_size(w.cache, b, 2, 4) > 0
    outs, graphs = [torch.empty_like(x) for x in want], []
    for q, o in zip(qs, outs):
        ws = torch.empty(bd.paged_attention_workspace_size(w.cache, b, 2, 4), dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            bd.paged_attention(w.cache, b, q, out=o, workspace=ws)
        graphs.append((g, ws))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(outs, want))
    s = streams[0]
    with torch.cuda.stream(s):
        o = bd.paged_attention(w.cache, b, qs[1])
    s.synchronize()
    assert torch.equal(o, want[1])
    o = bd.paged_attention(w.cache, b, qs[0], stream=torch.cuda.current_stream())
    assert torch.equal(o, want[0])


def test_captured_without_a_workspace_and_two_calls_at_once():
    """A capture takes its workspace from the graph's own pool; calls on two streams each get their own."""
    w = World(3, 2, 128, 64, torch.bfloat16, seed=44, max_tokens=3000)
    w.step([2900, 1500, 40])
    b = w.batch([1, 2, 1])
    qs = [to_device(queries(w.rng, 4, 8, 128, w.kind)[0], w.kind) for _ in range(3)]
    want = [bd.paged_attention(w.cache, b, q) for q in qs]
    x, out = qs[0].clone(), torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.paged_attention(w.cache, b, x, out=out)
    for q, y in zip(qs, want):
        x.copy_(q)
        junk = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
        graph.replay()
        assert torch.equal(out, y)
        del junk
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for q, s in zip(qs, streams):
            with torch.cuda.stream(s):
                got.append(bd.paged_attention(w.cache, b, q))
        torch.cuda.synchronize()
        assert all(torch.equal(g, y) for g, y in zip(got, want))
    got = [bd.paged_attention(w.cache, b, q, stream=s) for q, s in zip(qs, streams)]     # the stream as an argument
    torch.cuda.synchronize()
    assert all(torch.equal(g, y) for g, y in zip(got, want))
    bd.poll_status()


def test_the_tensor_core_product_and_the_chunk_kernel_back_to_back():
    """Both keep their accumulators in tensor memory and start under each other's tails."""
    w = World(1, 2, 128, 64, torch.bfloat16, seed=45, max_tokens=700)
    w.step([600])
    b = w.batch([200])
    q = to_device(queries(w.rng, 200, 8, 128, w.kind)[0], w.kind)
    rng = np.random.default_rng(1)
    wq = bd.quantize_weights(torch.from_numpy(rng.standard_normal((1024, 1024)).astype(np.float32)).cuda(), bd.SELECT_TWO_STAGE)
    want_o = bd.paged_attention(w.cache, b, q)
    want_y = bd.linear(want_o.view(200, 1024), wq)
    for _ in range(20):
        o = bd.paged_attention(w.cache, b, q)
        y = bd.linear(o.view(200, 1024), wq)
        assert torch.equal(bd.paged_attention(w.cache, b, q), want_o) and torch.equal(y, want_y) and torch.equal(o, want_o)
    bd.poll_status()
