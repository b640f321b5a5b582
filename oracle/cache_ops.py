"""Operators on a decoding batch's cache, one prompt at a time, in float64 straight from their definitions.

The decode stage of the paper (Section 2.1) attends to the keys and values of everything before a token; these are the
steps a server adds: several drafted tokens at once (each sees the context and some of the drafted tokens), running
attention weights per slot, the slots kept under a budget, and moving them together.
"""
import numpy as np


def scores(q, k, scale):
    """q [n, Hq, D], k [T, Hkv, D] -> [n, Hq, T]."""
    group = q.shape[1] // k.shape[1]
    kk = np.repeat(k.astype(np.float64), group, axis=1)
    with np.errstate(invalid="ignore", over="ignore"):
        return np.einsum("nhd,thd->nht", q.astype(np.float64), kk) * scale


def sees(n, ctx, node_mask=None):
    """[n, ctx + n]: what every node sees; node_mask [n, n] or None (nodes up to itself)."""
    nodes = np.tril(np.ones((n, n), dtype=bool)) if node_mask is None else np.asarray(node_mask, dtype=bool)
    return np.concatenate([np.ones((n, ctx), dtype=bool), nodes], axis=1)


def tree_attention(q, k, v, ctx, node_mask, scale):
    """Returns out [n, Hq, D], lse [n, Hq] and mean_abs, the same average of |v| (what rounding errors scale with)."""
    n, hq, d = q.shape
    x = scores(q, k, scale)
    seen = sees(n, ctx, node_mask)
    group = hq // k.shape[1]
    out, mean_abs = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse = np.full((n, hq), -np.inf)
    vv = v.astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for i in range(n):
            at = np.flatnonzero(seen[i])
            if len(at) == 0:
                continue
            for h in range(hq):
                s = x[i, h, at]
                top = np.max(s)
                e = np.exp(s - top)
                lse[i, h] = top + np.log(e.sum())
                out[i, h] = (e / e.sum()) @ vv[at, h // group]
                mean_abs[i, h] = (e / e.sum()) @ np.abs(vv[at, h // group])
    return out, lse, mean_abs


def attention_weights(q, k, lse, use, ctx, node_mask, scale, weights, decay):
    """weights [Hkv, ctx + n] after one step (rows with use, heads of each KV head)."""
    n, hq, _ = q.shape
    hkv = k.shape[1]
    x = scores(q, k, scale)
    seen = sees(n, ctx, node_mask)
    out = decay * weights.astype(np.float64) if decay != 0 else np.zeros(weights.shape)
    for i in range(n):
        if use is not None and not use[i]:
            continue
        for h in range(hq):
            if lse[i, h] == -np.inf:
                continue
            out[h // (hq // hkv), seen[i]] += np.exp(x[i, h, seen[i]] - float(lse[i, h]))
    return out


def select_slots(weights, length, budget, sink, recent):
    """Ascending kept slots of one head."""
    if length <= budget:
        return list(range(length))
    always = [s for s in range(length) if s < sink or s >= length - recent]
    w = np.where(np.isnan(weights[:length]), -np.inf, weights[:length])
    rest = sorted((s for s in range(sink, length - recent)), key=lambda s: (-w[s], s))
    return sorted(always + rest[:budget - len(always)])
