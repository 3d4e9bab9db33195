"""CPU oracle of a serving step over a paged cache (test infrastructure, like the rest of this package).

A sequence's storage is the KV cache of the appendix "Quantization Dimension" (oracle/kvcache.py), one per KV head; which
page holds what is the library's business and does not show in the values.  Attention here keeps queries and
probabilities in high precision (only the cache is in 4 bits); the rotation is the usual one on pairs of elements.  numpy, fp64.
"""
import numpy as np

from . import dequantize
from .kvcache import KVCache


class Sequence:
    """One sequence: a cache per KV head."""

    def __init__(self, kv_heads, head_dim, dtype):
        self.heads = [KVCache(head_dim, dtype) for _ in range(kv_heads)]

    @property
    def length(self):
        return self.heads[0].length

    def append(self, k_rows, v_rows):
        """[t, kv_heads, head_dim] source rows (fp32, or uint16 patterns)."""
        for h, c in enumerate(self.heads):
            c.append(k_rows[:, h], v_rows[:, h])

    def keys(self):
        """fp64 [kv_heads, length, head_dim]."""
        return np.stack([dequantize(*c.keys()) if c.length else np.zeros((0, c.d)) for c in self.heads]).astype(np.float64)

    def values(self):
        out = []
        for c in self.heads:
            stored = [dequantize(*ch).T for ch in c.chunks]
            out.append(np.concatenate(stored + [c.values_recent()], axis=0))
        return np.stack(out).astype(np.float64)


def attention(q, k, v, scale, softcap=0.0, window=0):
    """Causal attention of the last t tokens: q [t, q_heads, d], k and v [kv_heads, length, d] fp64.  Returns (o, lse, absolute
    weights' sums sum_j p_j |v_j|, sum_k |q_k| |k_k| maxima per row, sum of |v_j| over the visible j)."""
    t, heads, d = q.shape
    kv_heads, length = k.shape[:2]
    o, pv, qk, vv = (np.zeros((t, heads, d)) for _ in range(4))
    lse = np.full((t, heads), -np.inf)
    key = np.arange(length)
    for h in range(heads):
        kh, vh = k[h // (heads // kv_heads)], v[h // (heads // kv_heads)]
        for i in range(t):
            pos = length - t + i
            see = (key <= pos) & ((key > pos - window) if window else True)
            if not see.any():
                continue
            s = scale * (kh[see] @ q[i, h])
            if softcap:
                s = softcap * np.tanh(s / softcap)
            m = s.max()
            p = np.exp(s - m)
            lse[i, h] = m + np.log(p.sum())
            o[i, h] = p @ vh[see] / p.sum()
            pv[i, h] = p @ np.abs(vh[see]) / p.sum()
            qk[i, h] = (np.abs(kh[see]) @ np.abs(q[i, h])).max()
            vv[i, h] = np.abs(vh[see]).sum(0) / p.sum()
    return o, lse, pv, qk, vv


def norm_rope(x, weight, cos_sin, positions, eps, interleaved):
    """x [rows, heads, d] fp64; weight [d] or None; cos_sin [positions, rot]."""
    y = x.copy()
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight
    rot = cos_sin.shape[1]
    c, s = cos_sin[positions][:, None, : rot // 2], cos_sin[positions][:, None, rot // 2:]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    z = y.copy()
    z[..., a] = y[..., a] * c - y[..., b] * s
    z[..., b] = y[..., b] * c + y[..., a] * s
    return z
