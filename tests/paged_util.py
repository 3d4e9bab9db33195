"""Shared by the paged-cache tests: sequences with their oracle, a page allocator and a step's batch."""
import numpy as np
import torch

import paper_2501_01144_b200 as bd
from oracle.paged import Sequence
from paper_2501_01144_b200 import inputs
from util import ORACLE_DTYPE, to_device


def source_rows(rng, t, kv_heads, d, kind):
    """Keys with an outlier channel and values with uneven channels, in the bits of `kind`."""
    k = rng.standard_normal((t, kv_heads, d)).astype(np.float32)
    k[:, :, 5] *= 9.0
    v = (rng.standard_normal((t, kv_heads, d)) * np.exp2(np.arange(d) % 5 - 2)).astype(np.float32)
    if kind == torch.float32:
        return k, v
    conv = inputs.to_bf16_bits if kind == torch.bfloat16 else inputs.to_f16_bits
    return conv(k), conv(v)


def values_of(bits, kind):
    if kind == torch.float32:
        return np.asarray(bits, np.float64)
    if kind == torch.bfloat16:
        return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)
    return bits.view(np.float16).astype(np.float64)


class World:
    """n sequences in one cache, every unused byte of it set to 0xff (NaN rows in the tail, junk in the pool)."""

    def __init__(self, n, kv_heads, d, page, kind, seed, max_tokens, extra_pages=3):
        self.rng = np.random.default_rng(seed)
        self.n, self.kv_heads, self.d, self.page, self.kind = n, kv_heads, d, page, kind
        width = -(-max_tokens // page)
        order = self.rng.permutation(n * width + extra_pages)
        self.table = torch.tensor(order[: n * width].reshape(n, width).astype(np.int32)).cuda()
        self.slots = torch.tensor(self.rng.permutation(n + 2)[:n].astype(np.int32)).cuda()
        self.cache = bd.PagedKVCache(n * width + extra_pages, kv_heads, d, n + 2, page, kind)
        self.cache.pool.fill_(255)
        self.cache.tail.view(torch.uint8).fill_(255)
        self.seqs = [Sequence(kv_heads, d, ORACLE_DTYPE[kind]) for _ in range(n)]

    def lengths(self):
        return [s.length for s in self.seqs]

    def batch(self, new, kv_len=None):
        """Batch whose sequence i has new[i] rows; kv_len defaults to the oracle's lengths."""
        i32 = lambda x: torch.tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
        starts = np.concatenate([[0], np.cumsum(new)])
        return bd.PagedBatch(self.table, self.slots, i32(self.lengths() if kv_len is None else kv_len), i32(starts), int(max(new)))

    def step(self, new):
        """Append new[i] tokens to sequence i on both sides."""
        rows = [source_rows(self.rng, t, self.kv_heads, self.d, self.kind) for t in new]
        for s, (k, v) in zip(self.seqs, rows):
            s.append(k, v)
        b = self.batch(new)
        k, v = (np.concatenate([r[j] for r in rows]) for j in (0, 1))
        bd.paged_append(self.cache, b, to_device(k, self.kind), to_device(v, self.kind))
        return b, k, v
