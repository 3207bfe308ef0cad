"""Oracle of the operators for drafting over the cache (NumPy, float64).

Trees of drafted tokens: ``tree_mask`` (who sees whom, from the parents),
``tree_attention`` (softmax over the context and the visible nodes, with the weight
every slot receives), eviction: ``cache_select`` and ``cache_compact``, and a
sampler's rules: ``adjust_logits``.  Loops follow the definitions, one row at a time.
"""
from __future__ import annotations

import numpy as np

from .bf16 import round_bf16
from .decoder import rmsnorm, rope, silu


def tree_mask(parents):
    """parents [B, T] -> (sees [B, T, T] bool, depth [B, T])."""
    parents = np.asarray(parents)
    B, T = parents.shape
    sees = np.zeros((B, T, T), bool)
    depth = np.zeros((B, T), np.int32)
    for b in range(B):
        for t in range(T):
            u = t if parents[b, t] > -2 else -1
            while u >= 0:
                sees[b, t, u] = True
                u = parents[b, u]
                depth[b, t] += u >= 0
    return sees, depth


def pack_mask(sees):
    """[B, T, T] bool -> [B, T, ceil(T / 64)] int64 bits."""
    B, T, _ = sees.shape
    W = (T + 63) // 64
    words = np.zeros((B, T, W), np.uint64)
    for u in range(T):
        words[:, :, u // 64] |= sees[:, :, u].astype(np.uint64) << np.uint64(u % 64)
    return words.view(np.int64)


def tree_attention(q, k, v, lens, sees=None, n_nodes=None, scale=None, weights_in=None):
    """q [B, T, H, dh], k and v [B, cap, Hkv, dh] -> (out, weights [B, Hkv, cap]); rows of
    dead nodes and slots past the live nodes are NaN (the operator leaves them)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    B, T, H, dh = q.shape
    cap, Hkv = k.shape[1:3]
    G = H // Hkv
    scale = dh ** -0.5 if scale is None else scale
    out = np.full(q.shape, np.nan)
    weights = np.full((B, Hkv, cap), np.nan)
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        live = T if n_nodes is None else min(max(int(n_nodes[b]), 0), T)
        live = min(live, cap - n)
        for hk in range(Hkv):
            total = np.zeros(n + live)
            if weights_in is not None:
                total[:n] = weights_in[b, hk, :n]
            for t in range(live):
                nodes = np.arange(live)[sees[b, t, :live]] if sees is not None else np.arange(t + 1)
                at = np.concatenate([np.arange(n), n + nodes])
                for h in range(hk * G, hk * G + G):
                    if not len(at):
                        out[b, t, h] = 0.0
                        continue
                    s = scale * (k[b, at, hk] @ q[b, t, h])
                    e = np.exp(s - s.max())
                    p = e / e.sum()
                    out[b, t, h] = p @ v[b, at, hk]
                    total[at] += p
            weights[b, hk, :n + live] = total
    return out, weights


def cache_select(weights, lens, keep, n_first=0, n_last=0, shared=False):
    """weights [L, B, Hkv, cap] -> (idx [L, B, G, keep], new lens [B])."""
    w = np.asarray(weights, np.float32)
    L, B, Hkv, cap = w.shape
    if shared:
        s = np.zeros((L, B, 1, cap))
        for h in range(Hkv):
            s += w[:, :, h:h + 1].astype(np.float64)
        w = s.astype(np.float32)
    idx = np.full(w.shape[:3] + (keep,), -1, np.int32)
    new = np.zeros(B, np.int32)
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        new[b] = min(n, keep)
        for l in range(L):
            for g in range(w.shape[2]):
                x = w[l, b, g, :n].astype(np.float64)
                x[np.isnan(x)] = -np.inf
                always = np.zeros(n, bool)
                always[:n_first] = True
                always[max(0, n - n_last):] = True
                order = sorted(range(n), key=lambda j: (not always[j], -x[j], j))
                idx[l, b, g, :new[b]] = np.sort(order[:new[b]])
    return idx, new


def cache_compact(x_in, x_out, idx, count=None, base=None):
    """Rows of x_in [L, B, cap, Hkv, ...] into a copy of x_out; idx [1 or L, B, 1 or Hkv, n]."""
    out = x_out.copy()
    L, B, cap, Hkv = x_in.shape[:4]
    for l in range(L):
        for b in range(B):
            first = 0 if base is None else int(base[b])
            n = idx.shape[3] if count is None else min(max(int(count[b]), 0), idx.shape[3])
            for h in range(Hkv):
                row = idx[min(l, idx.shape[0] - 1), b, min(h, idx.shape[2] - 1)]
                for i in range(n):
                    src, dst = first + int(row[i]), first + i
                    if row[i] >= 0 and first >= 0 and src < cap and dst < out.shape[2]:
                        out[l, b, dst, h] = x_in[l, b, src, h]
    return out


def adjust_logits(logits, history=None, n_history=None, n_prompt=None, node_tokens=None, sees=None, repetition=None,
                  frequency=None, presence=None, bias_ids=None, bias=None, allowed=None, n_nodes=None):
    """logits [B, T, V] -> (adjusted float64, arg max int32); rows of dead nodes NaN and -2."""
    x = np.asarray(logits, np.float64)
    B, T, V = x.shape
    out = np.full(x.shape, np.nan)
    best = np.full((B, T), -2, np.int32)
    for b in range(B):
        live = T if n_nodes is None else min(max(int(n_nodes[b]), 0), T)
        for t in range(live):
            said, seen = np.zeros(V, np.int64), np.zeros(V, bool)
            if history is not None:
                n = min(max(int(n_history[b]), 0), history.shape[1])
                for i in range(n):
                    v = int(history[b, i])
                    if 0 <= v < V:
                        seen[v] = True
                        said[v] += i >= (0 if n_prompt is None else int(n_prompt[b]))
            if node_tokens is not None:
                for u in range(live):
                    v = int(node_tokens[b, u])
                    if (sees[b, t, u] if sees is not None else u <= t) and 0 <= v < V:
                        seen[v] = True
                        said[v] += 1
            y = x[b, t].copy()
            if repetition is not None:
                r = float(repetition[b])
                y[seen] = np.where(y[seen] > 0, y[seen] / r, y[seen] * r)
            f = 0.0 if frequency is None else float(frequency[b])
            p = 0.0 if presence is None else float(presence[b])
            y[said > 0] = y[said > 0] - f * said[said > 0] - p
            if bias_ids is not None:
                for v, w in zip(bias_ids[b], bias[b]):
                    if 0 <= v < V:
                        y[int(v)] += float(w)
            if allowed is not None:
                y[~np.broadcast_to(allowed, x.shape)[b, t]] = -np.inf
            out[b, t] = y
            z = np.where(np.isnan(y), -np.inf, y)
            best[b, t] = -1 if z.max() == -np.inf else int(np.argmax(z))
    return out, best


def decode_tree(x, weights, k, v, lens, pos, parents, cfg, recipe="bf16", attn_weights=None):
    """One step over the nodes x [B, T, d] of a tree on explicit caches k, v [L, B, cap, d]
    (updated in place, as are attn_weights [L, B, H, cap] if given) -> states [B, T, d]."""
    rnd = round_bf16 if recipe == "bf16" else (lambda t: t)
    get = weights if callable(weights) else (lambda l: weights[l])
    f = lambda a: np.asarray(a, np.float64)  # noqa: E731
    B, T, d = x.shape
    H, dh = cfg.H, cfg.d // cfg.H
    sees, depth = tree_mask(parents)
    live = [int((np.asarray(parents[b]) > -2).sum()) for b in range(B)]
    at = (np.asarray(pos)[:, None] + depth).reshape(-1)
    h = f(x).reshape(B * T, d).copy()
    for l in range(k.shape[0]):
        w = get(l)
        xn = f(rnd(rmsnorm(h, f(w["attn_norm"]), cfg.eps)))
        q, kk, vv = ((xn @ f(w[m]).T).reshape(B * T, H, dh) for m in ("wq", "wk", "wv"))
        q, kk, vv = f(rnd(rope(q, at, cfg.theta))), f(rnd(rope(kk, at, cfg.theta))), f(rnd(vv))
        for b in range(B):
            rows = slice(b * T, b * T + live[b])
            k[l, b, lens[b]:lens[b] + live[b]] = kk[rows].reshape(live[b], d)
            v[l, b, lens[b]:lens[b] + live[b]] = vv[rows].reshape(live[b], d)
        shape = k.shape[1:3] + (H, dh)
        o, aw = tree_attention(q.reshape(B, T, H, dh), k[l].reshape(shape), v[l].reshape(shape), lens, sees, live,
                               weights_in=None if attn_weights is None else attn_weights[l])
        if attn_weights is not None:
            attn_weights[l] = np.where(np.isnan(aw), attn_weights[l], aw)
        o = f(rnd(np.nan_to_num(o).reshape(B * T, d)))
        h = h + o @ f(w["wo"]).T
        xn = f(rnd(rmsnorm(h, f(w["ffn_norm"]), cfg.eps)))
        h = h + f(rnd(silu(xn @ f(w["wg"]).T) * (xn @ f(w["wu"]).T))) @ f(w["wd"]).T
    return h.reshape(B, T, d)
