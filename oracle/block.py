"""CPU oracle of a mixture-of-experts block and of the norms around a block (test infrastructure, like the rest of this package).

The block's arithmetic around the DialectFP4 products is the usual one of such models; the products themselves are this package's
dequantised operands in fp64.  numpy, fp64.
"""
import numpy as np


def route(logits, top_k, score="softmax", bias=None, groups=1, top_groups=1, group_top=2, renormalise=True, scale=1.0, valid=None):
    """logits fp64 [tokens, experts] -> (ids, weights) [tokens, top_k]; ids -1 and weights 0 where no expert is left."""
    tokens, experts = logits.shape
    ids, weights = np.full((tokens, top_k), -1, np.int64), np.zeros((tokens, top_k))
    for t in range(tokens if valid is None else max(0, min(tokens, valid))):
        x = np.where(np.isnan(logits[t]), -np.inf, np.minimum(logits[t], np.finfo(np.float32).max))
        with np.errstate(over="ignore"):
            if score == "sigmoid":
                s = 1 / (1 + np.exp(-x))
            else:
                s = np.where(np.isneginf(x), 0.0, np.exp(x - x.max())) if x.max() > -np.inf else np.zeros(experts)
                s = s / s.sum() if s.sum() > 0 else s
        key = x if bias is None else s + bias
        there = ~np.isneginf(x) & ~np.isnan(key) & ~np.isneginf(key)
        if groups > 1:
            of = np.where(there, s if bias is None else key, -np.inf).reshape(groups, -1)
            best = np.sort(of, 1)[:, ::-1][:, :group_top]
            value = np.where(np.isneginf(best[:, 0]), -np.inf, np.where(np.isneginf(best), 0.0, best).sum(1))
            kept = [g for g in np.argsort(-value, kind="stable")[:top_groups] if value[g] > -np.inf]
            there &= np.isin(np.arange(experts) // (experts // groups), kept)
        order = np.argsort(-np.where(there, key, -np.inf), kind="stable")
        chosen = [e for e in order if there[e]][:top_k]
        w = s[chosen]
        if renormalise and len(chosen):
            if score == "softmax":                                # the same quotient, without underflow of all
                w = np.exp(x[chosen] - x[chosen].max())
            w = w / w.sum() if w.sum() > 0 else w * 0
        ids[t, : len(chosen)], weights[t, : len(chosen)] = chosen, w * scale
    return ids, weights


def plan(ids, experts):
    """(count, start, place): expert e's rows in the order of its tokens, starts at multiples of 128; a token has one row per expert."""
    tokens = [sorted({t for t in range(ids.shape[0]) if e in ids[t]}) for e in range(experts)]
    count = np.array([len(x) for x in tokens])
    start = np.concatenate([[0], np.cumsum((count + 127) // 128 * 128)])
    place = np.full(ids.shape, -1)
    for t in range(ids.shape[0]):
        for j, e in enumerate(ids[t]):
            if 0 <= e < experts:
                place[t, j] = start[e] + tokens[e].index(t)
    return count, start, place


def gated_order(inter):
    """Rows of the stored first product as rows of [gate; up]: in turns of 32."""
    r = np.arange(2 * inter)
    return r // 64 * 32 + r % 32 + np.where(r % 64 >= 32, inter, 0)


def activate(x, act):
    a = x if act == "silu" else 2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)
    with np.errstate(over="ignore"):
        return x / (1 + np.exp(-a))


def norm(x, weight, bias, layer, eps, offset):
    if layer:
        x = x - x.mean(-1, keepdims=True)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (weight + offset)
    return y if bias is None else y + bias
