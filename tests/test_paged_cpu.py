"""Paged cache without a GPU: the storage's index arithmetic (compiled for the host from the kernels' own header), the
refusals of the C entry points, and the oracle's pins."""
import copy
import ctypes
import os
import pickle
import subprocess
import types

import numpy as np
import pytest
import torch

import oracle
import paper_2501_01144_b200 as bd
from oracle.paged import Sequence, attention, norm_rope

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HARNESS = r"""
#include "paged_common.cuh"
using namespace bd::pg;
extern "C" {
int word(int b, int r, int t) { return word_byte(b, r, t); }
int entry(int nb, int b, int r) { return entry_of(nb, b, r); }
int row(int token) { return key_row(token); }
int token(int row) { return key_token(row); }
long long record(const int *table, long long ld, int pages, int heads, int per_page, int d, int i, int h, int c) {
    Pool p{}; p.pages = pages; p.kv_heads = heads; p.chunks_per_page = per_page; p.head_dim = d;
    Batch b{}; b.table = table; b.ld_table = ld;
    return record_offset(p, b, i, h, c);
}
long long tail(int heads, int d, int slot, int h, int token) {
    Pool p{}; p.kv_heads = heads; p.head_dim = d;
    return tail_offset(p, slot, h, token);
}
int sequence(const int *kv, const int *start, int i, int rows, int max_q, int max_kv, int *out) {
    Batch b{}; b.kv_len = kv; b.q_start = start; b.rows = rows; b.max_q = max_q; b.max_kv = max_kv;
    Sequence s = sequence_of(b, i);
    out[0] = s.q0; out[1] = s.t; out[2] = s.kv;
    return s.ok;
}
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    (d / "h.cpp").write_text(HARNESS)
    so = d / "h.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2501_01144_b200", "csrc"), "-o", str(so), str(d / "h.cpp")], check=True)
    lib = ctypes.CDLL(str(so))
    lib.record.restype = lib.tail.restype = ctypes.c_longlong
    lib.record.argtypes = [ctypes.c_void_p, ctypes.c_longlong] + [ctypes.c_int] * 7
    lib.sequence.argtypes = [ctypes.c_void_p, ctypes.c_void_p] + [ctypes.c_int] * 4 + [ctypes.c_void_p]
    return lib


@pytest.mark.parametrize("nb", [2, 4])
def test_every_word_and_entry_of_a_tile_has_a_place_of_its_own(host, nb):
    words = {host.word(b, r, t) for b in range(nb) for r in range(32) for t in range(4)}
    assert words == set(range(0, 512 * nb, 4))
    assert {host.entry(nb, b, r) for b in range(nb) for r in range(32)} == set(range(32 * nb))
    assert sorted(host.row(k) for k in range(32)) == list(range(32))
    assert all(host.token(host.row(k)) == k for k in range(32))
    # the entries of one token (one row, all tiles) are neighbours: whole bytes, shared with no other token
    for r in range(32):
        e = sorted(host.entry(nb, b, r) for b in range(nb))
        assert e == list(range(e[0], e[0] + nb)) and e[0] % nb == 0


def test_offsets_pass_32_bits_and_pages_outside_the_pool_are_told(host):
    table = np.array([[7, 2_000_000], [-1, 3], [2_000_001, 2_147_483_647]], np.int32)
    rec = lambda i, h, c: host.record(table.ctypes.data, 2, 2_000_001, 8, 2, 128, i, h, c)  # noqa: E731
    assert rec(0, 0, 0) == 7 * 8 * 2 * 4480 and rec(0, 3, 1) == ((7 * 8 + 3) * 2 + 1) * 4480
    assert rec(0, 7, 3) == ((2_000_000 * 8 + 7) * 2 + 1) * 4480 > 2 ** 36
    assert rec(1, 0, 0) == -1 and rec(1, 0, 2) == 3 * 16 * 4480
    assert rec(2, 0, 0) == -1 and rec(2, 0, 3) == -1
    assert host.tail(8, 128, 300_000, 7, 77) == ((300_000 * 8 + 7) * 64 + 13) * 128 > 2 ** 33


def test_sequences_that_contradict_the_bounds_are_told(host):
    out = (ctypes.c_int * 3)()

    def seq(kv, a, b, rows=10, max_q=4, max_kv=100):
        k, s = np.array([kv], np.int32), np.array([a, b], np.int32)
        return host.sequence(k.ctypes.data, s.ctypes.data, 0, rows, max_q, max_kv, out), tuple(out)

    assert seq(50, 2, 5) == (1, (2, 3, 50))
    assert seq(0, 0, 0)[0] == 1 and seq(100, 6, 10)[0] == 1
    for bad in ((50, -1, 2), (50, 5, 4), (50, 7, 11), (50, 0, 5), (-1, 0, 1), (101, 0, 1), (50, -2_147_483_648, 2_147_483_647)):
        assert seq(*bad) == (0, (0, 0, 0))


# ---- refusals: everything below returns before any launch, so made-up aligned addresses do ----

C, B, R = bd.binding._CPagedCache, bd.binding._CPagedBatch, bd.binding._CRopeOperand


def cache(**kw):
    a = dict(pool=0x1000, tail=0x2000, dtype=bd.BF16, pages=10, slots=4, kv_heads=2, page_tokens=64, head_dim=128)
    a.update(kw)
    return C(*a.values())


def batch(**kw):
    a = dict(page_table=0x1000, slot=0x2000, kv_len=0x3000, q_start=0x4000, ld_table=5, n=3, rows=6, max_q=2, max_kv=320)
    a.update(kw)
    return B(*a.values())


BAD_COMMON = [
    (dict(pool=0), {}, 1), (dict(tail=0), {}, 1), (dict(dtype=5), {}, 1), (dict(pages=0), {}, 1), (dict(kv_heads=-1), {}, 1),
    (dict(head_dim=96), {}, 2), (dict(head_dim=256), {}, 2), (dict(page_tokens=48), {}, 2), (dict(page_tokens=0), {}, 2),
    (dict(pool=0x1008), {}, 3), (dict(tail=0x2004), {}, 3), (dict(pages=2 ** 31), {}, 4), (dict(kv_heads=70000), {}, 4),
    ({}, dict(page_table=0), 1), ({}, dict(kv_len=0), 1), ({}, dict(n=0), 1), ({}, dict(rows=-1), 1), ({}, dict(max_q=-1), 1),
    ({}, dict(max_q=7), 2), ({}, dict(max_kv=321), 2), ({}, dict(n=65536), 4), ({}, dict(q_start=0x4002), 3), ({}, dict(max_kv=2 ** 31, ld_table=2 ** 40), 4),
]


@pytest.mark.parametrize("c,b,status", BAD_COMMON)
def test_bad_caches_and_batches_are_refused(c, b, status):
    lib = bd.load()
    cc, bb = cache(**c), batch(**b)
    rc, rb = ctypes.byref(cc), ctypes.byref(bb)
    hd = cc.head_dim
    assert lib.bd_paged_append(rc, rb, 0x8000, 0x9000, 4 * hd, hd, 4 * hd, hd, None) == status
    assert lib.bd_paged_read(rc, rb, 0x8000, 0x9000, 4 * hd, hd, 4 * hd, hd, None) == status
    assert lib.bd_paged_attention(rc, rb, 0x8000, 4, 4 * hd, hd, 0.1, 0.0, 0, 0x9000, bd.BF16, 4 * hd, hd, None, 0x100000, 1 << 40, None) == status


def test_null_structures_are_refused():
    lib = bd.load()
    cc, bb = cache(), batch()
    assert lib.bd_paged_append(None, ctypes.byref(bb), 0x8000, 0x9000, 256, 128, 256, 128, None) == 1
    assert lib.bd_paged_append(ctypes.byref(cc), None, 0x8000, 0x9000, 256, 128, 256, 128, None) == 1
    assert lib.bd_paged_sizes(None, None, None) == 1
    assert lib.bd_qk_norm_rope(None, None, bd.BF16, 1, 128, 0x1000, 0x2000, 10, 128, 0, 1e-6, None) == 1


@pytest.mark.parametrize("args,status", [
    ((0, 0x9000, 256, 128, 256, 128), 1), ((0x8000, 0, 256, 128, 256, 128), 1), ((0x8000, 0x9000, 128, 128, 256, 128), 2),
    ((0x8000, 0x9000, 256, 64, 256, 128), 2), ((0x8000, 0x9000, 0, 128, 256, 128), 2), ((0x8002, 0x9000, 256, 128, 256, 128), 3),
    ((0x8000, 0x9000, 260, 128, 256, 128), 3), ((0x8000, 0x9000, 256, 132, 264, 132), 2), ((0x8000, 0x9000, 512, 256, 264, 132), 3),
])
def test_bad_rows_are_refused(args, status):
    lib = bd.load()
    cc, bb = cache(), batch()
    assert lib.bd_paged_append(ctypes.byref(cc), ctypes.byref(bb), *args, None) == status
    assert lib.bd_paged_read(ctypes.byref(cc), ctypes.byref(bb), *args, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q_heads=3), 2), (dict(q_heads=0), 1), (dict(window=-1), 1), (dict(softcap=-1.0), 1), (dict(softcap=float("nan")), 1), (dict(softcap=1e-9), 1), (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1),
    (dict(odtype=9), 1), (dict(odtype=bd.F16), 4), (dict(dtype=bd.F32), 4), (dict(ldo=500), 2), (dict(lse=0x5002), 3), (dict(ws=0, q_heads=4), 8),
    (dict(ws=0x100010, q_heads=4), 3), (dict(wbytes=100), 8),
])
def test_bad_attention_calls_are_refused(kw, status):
    lib = bd.load()
    a = dict(q_heads=4, scale=0.1, softcap=0.0, window=0, odtype=bd.BF16, ldo=512, lse=None, ws=0x100000, wbytes=1 << 40, dtype=bd.BF16)
    a.update(kw)
    cc, bb = cache(dtype=a["dtype"]), batch(ld_table=100, max_kv=6400)      # long enough to be shared out: a workspace is needed
    assert lib.bd_paged_attention(ctypes.byref(cc), ctypes.byref(bb), 0x8000, a["q_heads"], 512, 128, a["scale"], a["softcap"], a["window"], 0x9000, a["odtype"],
                                  a["ldo"], 128, a["lse"], a["ws"], a["wbytes"], None) == status


@pytest.mark.parametrize("b,q_heads", [
    (dict(rows=2 ** 31 - 1, max_q=2 ** 31 - 1), 1), (dict(rows=2 ** 30, max_q=2 ** 30), 2), (dict(rows=2 ** 30, max_q=2 ** 30), 2 ** 62),
    (dict(max_kv=2 ** 31 - 40, ld_table=2 ** 26), 1)])
def test_sizes_that_pass_32_bits_are_refused(b, q_heads):
    lib = bd.load()
    cc, bb = cache(kv_heads=1), batch(n=1, **b)
    assert lib.bd_paged_attention(ctypes.byref(cc), ctypes.byref(bb), 0x8000, q_heads, 128 * q_heads if q_heads < 2 ** 40 else 128, 128, 0.1, 0.0, 0, 0x9000, bd.BF16,
                                  128 * q_heads if q_heads < 2 ** 40 else 128, 128, None, None, 0, None) == 4


@pytest.mark.parametrize("kw,status", [
    (dict(rot=24), 2), (dict(rot=0), 2), (dict(rot=144), 2), (dict(head_dim=96), 2), (dict(dtype=7), 1), (dict(positions=0), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(pos=0), 1), (dict(table=0), 1), (dict(table=0x2004), 3), (dict(heads=0), 1), (dict(x=0x8004), 3), (dict(ldx=128), 2), (dict(w=0x7004), 3),
])
def test_bad_rotations_are_refused(kw, status):
    lib = bd.load()
    a = dict(dtype=bd.BF16, head_dim=128, pos=0x1000, table=0x2000, positions=16, rot=128, eps=1e-6, heads=2, x=0x8000, ldx=256, w=0)
    a.update(kw)
    q, k = R(a["x"], 0x9000, a["w"], a["heads"], a["ldx"], 128, 256, 128), R(0, 0, 0, 0, 0, 0, 0, 0)
    assert lib.bd_qk_norm_rope(ctypes.byref(q), ctypes.byref(k), a["dtype"], 5, a["head_dim"], a["pos"], a["table"], a["positions"], a["rot"], 0, a["eps"], None) == status


def test_sizes():
    lib = bd.load()
    p, t = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.bd_paged_sizes(ctypes.byref(cache()), ctypes.byref(p), ctypes.byref(t)) == 0
    assert p.value == 10 * 2 * 2 * 35 * 128 and t.value == 4 * 2 * 64 * 128 * 2
    assert lib.bd_paged_sizes(ctypes.byref(cache(head_dim=32)), None, None) == 2
    assert lib.bd_status_string(10) != b"unknown status"


# ---- the descriptors that Python keeps ----


@pytest.mark.parametrize("duplicate", [copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x)), copy.copy], ids=["deepcopy", "pickle", "copy"])
def test_a_copied_cache_or_batch_is_described_by_its_own_tensors(monkeypatch, duplicate):
    """The descriptor holds addresses: a copy that kept it would read and write the original's buffers, or freed ones."""
    where = lambda *members: tuple(x.data_ptr() if torch.is_tensor(x) else x for x in members)  # noqa: E731
    monkeypatch.setattr(bd.binding, "_paged", types.SimpleNamespace(cache=where, batch=where))
    i32 = lambda *s: torch.arange(int(np.prod(s)), dtype=torch.int32).view(*s)  # noqa: E731
    cache = bd.PagedKVCache.from_buffers(torch.ones(3, 2, 1, 35 * 64, dtype=torch.uint8), torch.ones(2, 2, 64, 64), 32)
    batch = bd.PagedBatch(i32(2, 3), i32(2), i32(2), i32(3), 4, max_kv=90)
    for x, names in ((cache, ("pool", "tail", "page_tokens")), (batch, ("page_table", "slots", "kv_len", "q_start", "max_q", "max_kv"))):
        y = duplicate(x)
        assert type(y) is type(x) and y._c == where(*(getattr(y, n) for n in names))
        for n in names:
            a, b = getattr(x, n), getattr(y, n)
            assert torch.equal(a, b) and (a.data_ptr() == b.data_ptr()) == (duplicate is copy.copy) if torch.is_tensor(a) else a == b
        with pytest.raises(AttributeError):
            setattr(y, names[0], None)


# ---- the oracle ----

def test_oracle_sequence_equals_its_source_on_the_grid():
    """Rows whose blocks are exactly representable come back unchanged, whole chunks and remainder alike."""
    d, n = 64, 45
    rng = np.random.default_rng(1)
    grid = np.array([0, .5, 1, 1.5, 2, 3, 4, 6], np.float32)          # the FP4 E2M1 dialect, maximum 6
    x = grid[rng.integers(0, 8, (n, 2, d))] * rng.choice([-1, 1], (n, 2, d)).astype(np.float32)
    x[:, :, ::32] = 6.0                                               # every key block has the dialect's maximum ...
    s = Sequence(2, d, oracle.F32)
    s.append(x[:20], x[:20])
    s.append(x[20:], x[20:])
    assert s.length == n and s.values().shape == (2, n, d)
    k = s.keys().transpose(1, 0, 2)
    on_grid = np.isclose(np.abs(k[..., None]), np.abs(x[..., None])).all()
    err = np.abs(k - x)
    assert on_grid or err.max() <= 1.0                                # (the dialect pair of 6 also holds 4.5 | 4.0)
    assert np.array_equal(s.values().transpose(1, 0, 2)[32:], x[32:])  # the remainder is the source


def test_oracle_attention_on_cases_with_a_known_answer():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((1, 9, 4)), rng.standard_normal((1, 9, 4))
    o, lse, *_ = attention(np.zeros((3, 2, 4)), k, v, 0.5)            # all scores equal: means over what is visible
    for i in range(3):
        assert np.allclose(o[i], v[0, : 7 + i].mean(0)) and np.allclose(lse[i], np.log(7 + i))
    o, *_ = attention(np.zeros((3, 2, 4)), k, v, 0.5, window=2)
    assert np.allclose(o[0], v[0, 5:7].mean(0))
    o, *_ = attention(1e3 * k[0, 8][None, None], k, v, 1.0, softcap=1e-9)   # a cap at zero: uniform again
    assert np.allclose(o[0, 0], v[0].mean(0))
    o, lse, *_ = attention(np.zeros((4, 1, 4)), k[:, :2], v[:, :2], 1.0)     # rows before the first token see nothing
    assert (o[:2] == 0).all() and np.isinf(lse[:2]).all() and np.allclose(o[2], v[0, 0])


def test_oracle_rotation_keeps_lengths_and_composes():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 3, 64))
    ang = np.arange(20)[:, None] * 0.1 ** (np.arange(16) / 16)
    tab = np.concatenate([np.cos(ang), np.sin(ang)], 1)
    for il in (False, True):
        y = norm_rope(x, None, tab, np.array([0, 1, 2, 7, 9]), 0.0, il)
        assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1)) and np.array_equal(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
        z = norm_rope(norm_rope(x, None, tab, np.full(5, 3), 0.0, il), None, tab, np.full(5, 4), 0.0, il)
        assert np.allclose(z, norm_rope(x, None, tab, np.full(5, 7), 0.0, il))
    y = norm_rope(x, np.ones(64), tab, np.zeros(5, int), 0.0, False)
    assert np.allclose((y * y).mean(-1), 1.0)
