"""Oracle of the operators over a paged cache (NumPy, float64).

Rotary positions with several axes: ``rope_axes`` and ``rope_append`` (with the pages it
writes), ``paged_attention`` of chunks of new tokens, ``pages_fork`` (the next step's page
tables) and ``beam_select``.  Loops follow the definitions, one row at a time.
"""
from __future__ import annotations

import numpy as np


def rope_axes(rot, theta, sections, interleaved=False):
    half, n = rot // 2, len(sections)
    assert sum(sections) == half
    freq = np.array([theta ** (-2.0 * i / rot) for i in range(half)])
    left, axis = list(sections), []
    for i in range(half):
        a = next(x for x in range(n) if left[x]) if not interleaved else (i % n if left[i % n] else 0)
        left[a] -= 1
        axis.append(a)
    assert min(left) == 0 and max(left) == 0
    return freq, np.array(axis, np.uint8)


def rows_of(lens, cu, N, slots):
    """[(row, sequence, position)] of the rows that belong to a sequence."""
    cu = [min(max(int(c), 0), N) for c in cu]
    out = []
    for b, n in enumerate(lens):
        n = min(max(int(n), 0), slots)
        out += [(r, b, n - (cu[b + 1] - r)) for r in range(cu[b], cu[b + 1])]
    return out


def page_of(table, b, i, n_pages):
    p = int(table[b, i])
    return p if 0 <= p < n_pages else -1


def turn(x, pos, freq, axis):
    """x [.., dh] of one token turned by the positions pos [n_axes]."""
    half = len(freq)
    a = np.array([float(pos[min(int(ax), len(pos) - 1)]) for ax in axis]) * freq
    y = np.array(x, np.float64)
    u, w = y[..., :half].copy(), y[..., half:2 * half].copy()
    y[..., :half] = u * np.cos(a) - w * np.sin(a)
    y[..., half:2 * half] = w * np.cos(a) + u * np.sin(a)
    return y


def rope_append(pos, freq, axis, q, k, v, k_pages, v_pages, table, lens, cu):
    """-> (q, k_pages, v_pages) after the call; rows of no sequence are NaN in q."""
    N, P = pos.shape[1], k_pages.shape[1]
    qo = np.full(q.shape, np.nan)
    kp, vp = np.array(k_pages, np.float64), np.array(v_pages, np.float64)
    for r, b, p in rows_of(lens, cu, N, table.shape[1] * P):
        qo[r] = turn(q[r], pos[:, r], freq, axis)
        page = page_of(table, b, p // P, len(kp)) if p >= 0 else -1
        if page >= 0:
            kp[page, p % P] = turn(k[r], pos[:, r], freq, axis)
            vp[page, p % P] = v[r]
    return qo, kp, vp


def paged_attention(q, k_pages, v_pages, table, lens, cu, window=0, scale=None):
    """-> (out [N, H, dh], spread, size, reach): rows of no sequence are NaN.  Of each output,
    spread = sum_j p_j |v_j - out| and size = sum_j p_j |v_j|; of each row and head, reach = (the
    largest sum of |scale q_c k_c| over its slots, their number)."""
    q, k_pages, v_pages = (np.asarray(x, np.float64) for x in (q, k_pages, v_pages))
    N, H, dh = q.shape
    P, Hkv = k_pages.shape[1:3]
    scale = dh ** -0.5 if scale is None else scale
    out, spread, size = (np.full(q.shape, np.nan) for _ in range(3))
    reach = np.zeros((N, H, 2))
    for r, b, p in rows_of(lens, cu, N, table.shape[1] * P):
        lo = max(0, p - window + 1) if window else 0
        at = [(page_of(table, b, j // P, len(k_pages)), j % P) for j in range(lo, p + 1)]
        at = np.array([x for x in at if x[0] >= 0], int).reshape(-1, 2)
        for h in range(H):
            if not len(at):
                out[r, h] = spread[r, h] = size[r, h] = 0.0
                continue
            K, V = k_pages[at[:, 0], at[:, 1], h // (H // Hkv)], v_pages[at[:, 0], at[:, 1], h // (H // Hkv)]
            s = scale * (K @ q[r, h])
            e = np.exp(s - s.max())
            w = e / e.sum()
            out[r, h] = w @ V
            spread[r, h] = w @ np.abs(V - out[r, h])
            size[r, h] = w @ np.abs(V)
            reach[r, h] = (abs(scale) * (np.abs(K) @ np.abs(q[r, h])).max(), len(at))
    return out, spread, size, reach


def pages_fork(table, lens, ref, parent, n_new, P):
    """-> (table, lens, ref, missing, copies [(page, its copy, slots)])."""
    B_in, M = table.shape
    ref = np.array(ref, np.int64)
    n_pages = len(ref)
    old = [min(max(int(n), 0), M * P) for n in lens]
    held = lambda b, i: page_of(table, b, i, n_pages)
    rows, n = [], []
    for b, p in enumerate(parent):
        ok = 0 <= p < B_in
        n.append(old[p] if ok else 0)
        rows.append([held(p, i) for i in range(-(-n[b] // P))])
    for b in range(B_in):
        for i in range(-(-old[b] // P)):
            if held(b, i) >= 0:
                ref[held(b, i)] -= 1
    for row in rows:
        for page in row:
            if page >= 0:
                ref[page] += 1
    grown = [min(n[b] + max(int(n_new[b]) if n_new is not None else 0, 0), M * P) if 0 <= parent[b] < B_in else 0 for b in range(len(parent))]
    writers = {}
    for b, row in enumerate(rows):
        if grown[b] > n[b] and n[b] % P and row[-1] >= 0:
            writers.setdefault(row[-1], []).append(b)
    copies_of = {}
    for page, who in writers.items():
        for b in (who if ref[page] > len(who) else who[1:]):
            copies_of[b] = page
    for page in copies_of.values():
        ref[page] -= 1
    free = [p for p in range(n_pages) if ref[p] <= 0]
    missing, copies = 0, []
    for b, row in enumerate(rows):
        def take():
            nonlocal missing
            if not free:
                missing += 1
                return -1
            ref[free[0]] = 1
            return free.pop(0)
        if b in copies_of:
            row[-1] = take()
            if row[-1] >= 0:
                copies.append((copies_of[b], row[-1], n[b] % P))
        row += [take() for _ in range(-(-grown[b] // P) - len(row))]
    out = np.full((len(parent), M), -1, np.int32)
    for b, row in enumerate(rows):
        out[b, :len(row)] = row
    return out, np.array(grown, np.int32), ref.astype(np.int32), missing, copies


def beam_select(logits, scores, n_out, done=None, eos=-1, history=None, n_history=None, history_out=None):
    """-> dict of scores, parent, token, done [B, n_out] and, with a history, its rows and lengths."""
    x, scores = np.asarray(logits, np.float64), np.asarray(scores, np.float64)
    B, K, V = x.shape
    res = {"scores": np.full((B, n_out), -np.inf), "parent": np.full((B, n_out), -1), "token": np.full((B, n_out), -1),
           "done": np.ones((B, n_out), int)}
    for b in range(B):
        cand = []
        for k in range(K):
            if not np.isfinite(scores[b, k]):
                continue
            if done is not None and done[b, k]:
                cand.append((-scores[b, k], k, 0, eos))
                continue
            row = np.where(np.isnan(x[b, k]), -np.inf, x[b, k])
            top = row.max()
            if not np.isfinite(top):
                continue
            lse = top + np.log(np.exp(row - top).sum())
            order = [v for v in np.argsort(-row, kind="stable")[:n_out] if row[v] > -np.inf]
            cand += [(-(scores[b, k] + (row[v] - lse)), k, i, v) for i, v in enumerate(order)]
        for i, (c, k, _, v) in enumerate(sorted(cand)[:n_out]):
            res["scores"][b, i], res["parent"][b, i], res["token"][b, i] = -c, b * K + k, v
            res["done"][b, i] = int((done is not None and done[b, k] != 0) or (eos >= 0 and v == eos))
    if history is not None:
        cap = history.shape[1]
        res["history"], res["n_history"] = np.array(history_out), np.zeros(B * n_out, int)
        for r, (p, v) in enumerate(zip(res["parent"].ravel(), res["token"].ravel())):
            if p < 0:
                continue
            n = min(max(int(n_history[p]), 0), cap)
            res["history"][r, :n] = history[p, :n]
            if n < cap and not (done is not None and done.ravel()[p]):
                res["history"][r, n] = v
                n += 1
            res["n_history"][r] = n
    return res
