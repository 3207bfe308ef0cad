"""The operators over a paged cache as a search uses them: prompts fed in chunks, rotary positions of three axes stored
into pages, attention over them, beams chosen, continued, copied and freed, against a search in 64 bits that recomputes
every hypothesis from its tokens."""
import numpy as np
import pytest
import torch

from gpu_common import need_gpu
from oracle import paged as op
from paged_common import f64, ints

pytestmark = pytest.mark.gpu
V, D, H, HKV, DH, L, P = 97, 64, 4, 2, 32, 2, 8


def weights(rng):
    w = lambda *s: rng.standard_normal(s) / np.sqrt(s[-1])
    layers = [dict(q=w(H * DH, D), k=w(HKV * DH, D), v=w(HKV * DH, D), o=w(D, H * DH)) for _ in range(L)]
    f32 = lambda x: x.astype(np.float32).astype(np.float64)
    return f32(2.0 * rng.standard_normal((V, D))), [{k: f32(v) for k, v in x.items()} for x in layers], f32(w(V, D) * 1.5)


def positions(i, grid):
    """Token i: text counts in all axes alike; the grid's tokens share their time and have a row and a column."""
    return (i, i, i) if i >= grid else (0, i // 4, i % 4)


def logits_of(tokens, grid, W, freq, axis, window):
    """Last logits of a hypothesis, from scratch."""
    emb, layers, head = W
    x = emb[tokens]
    n = len(tokens)
    turn = lambda y: np.stack([op.turn(y[i], positions(i, grid), freq, axis) for i in range(n)])
    for w in layers:
        q, k, v = turn((x @ w["q"].T).reshape(n, H, DH)), turn((x @ w["k"].T).reshape(n, HKV, DH)), (x @ w["v"].T).reshape(n, HKV, DH)
        out = np.zeros((n, H, DH))
        for i in range(n):
            lo = max(0, i - window + 1) if window else 0
            for h in range(H):
                s = k[lo:i + 1, h // (H // HKV)] @ q[i, h] / np.sqrt(DH)
                e = np.exp(s - s.max())
                out[i, h] = (e / e.sum()) @ v[lo:i + 1, h // (H // HKV)]
        x = x + out.reshape(n, -1) @ w["o"].T
    return x[-1] @ head.T


@pytest.mark.parametrize("seed,K,window", [(0, 4, 0), (1, 3, 7), (2, 5, 0)])
def test_search(seed, K, window):
    lib = need_gpu()
    rng = np.random.default_rng(seed)
    W = weights(rng)
    freq, axis = lib.rope_axes(DH, 10000.0, [6, 5, 5], True)
    B, steps, grid, M, n_pages = 3, 7, 8, 8, 90
    prompts = [rng.integers(0, V, n) for n in (17, 9, 24)]
    # the end is the first prompt's second best token: that beam ends at once
    eos = int(np.argsort(logits_of(prompts[0], grid, W, freq, axis, window))[-2])
    dev = lambda x: torch.from_numpy(np.asarray(x, np.float32)).cuda()
    emb, layers, head = dev(W[0]), [{k: dev(v) for k, v in x.items()} for x in W[1]], dev(W[2])
    df, da = torch.from_numpy(freq).cuda(), torch.from_numpy(axis).cuda()
    kp, vp = (torch.full((L, n_pages, P, HKV, DH), float("nan"), device="cuda") for _ in range(2))

    def model(tokens, pos, table, lens, cu, N):
        """Rows of the live sequences, packed, in a batch of N rows of which the last may be nobody's."""
        n = len(tokens)
        x = torch.zeros(N, D, device="cuda")
        x[:n] = emb[torch.as_tensor(tokens).cuda()]
        p = ints(np.concatenate([np.array(pos, int).T, np.zeros((3, N - n), int)], 1))
        for i, w in enumerate(layers):
            q, k, v = (x @ w[c].t() for c in "qkv")
            q = q.view(N, H, DH)
            lib.rope_append(p, df, da, q=q, q_out=q, k=k.view(N, HKV, DH), v=v.view(N, HKV, DH), k_pages=kp[i], v_pages=vp[i], table=table, lens=lens, cu_q=cu)
            out = torch.zeros(N, H, DH, device="cuda")
            lib.paged_attention(q, kp[i], vp[i], table, lens, cu, window=window, out=out)
            x = x + out.view(N, -1) @ w["o"].t()
        return x @ head.t()

    # the prompts in two chunks
    table, lens, ref = ints(np.full((B, M), -1)), ints([0] * B), ints(np.zeros(n_pages))
    done_tokens = [0] * B
    for part in (0.4, 1.0):
        news = [int(len(p) * part) - d for p, d in zip(prompts, done_tokens)]
        table, lens, ref, missing = lib.pages_fork(kp, vp, table, lens, ref, ints(range(B)), n_new=ints(news))
        cu = np.concatenate([[0], np.cumsum(news)])
        rows = [(p[i], positions(i, grid)) for p, d, n in zip(prompts, done_tokens, news) for i in range(d, d + n)]
        out = model([r[0] for r in rows], [r[1] for r in rows], table, lens, ints(cu), len(rows))
        done_tokens = [d + n for d, n in zip(done_tokens, news)]
    logits = out[torch.as_tensor(cu[1:] - 1).cuda()].view(B, 1, V)

    history = ints(np.zeros((B, 64)))
    n_history = ints([len(p) for p in prompts])
    for b, p in enumerate(prompts):
        history[b, :len(p)] = ints(p)
    scores, done = torch.zeros(B, 1, device="cuda"), None
    hyp = [[(0.0, list(p), False)] for p in prompts]
    for step in range(steps):
        best = lib.beam_select(logits, scores, K, done=done, eos=eos, history=history, n_history=n_history)
        # the same choice in 64 bits
        for b in range(B):
            x = np.stack([np.zeros(V) if d else logits_of(np.array(t), grid, W, freq, axis, window) for _, t, d in hyp[b]])[None]
            want = op.beam_select(x, np.array([[s for s, _, _ in hyp[b]]]), K, np.array([[int(d) for _, _, d in hyp[b]]]), eos)
            hyp[b] = [(want["scores"][0, i], hyp[b][want["parent"][0, i]][1] + ([] if hyp[b][want["parent"][0, i]][2] else [want["token"][0, i]]),
                       bool(want["done"][0, i])) for i in range(K)]
        got_h, got_n = best["history"].cpu().numpy(), best["n_history"].cpu().numpy()
        for b in range(B):
            for i, (s, t, d) in enumerate(hyp[b]):
                assert got_h[b * K + i, :got_n[b * K + i]].tolist() == list(t)
                assert bool(best["done"][b, i]) == d
                assert abs(best["scores"][b, i].item() - s) < 1e-4
        scores, done, history, n_history = best["scores"], best["done"], best["history"], best["n_history"]
        n_new = 1 - done.view(-1)
        table, lens, ref, missing = lib.pages_fork(kp, vp, table, lens, ref, best["parent"].view(-1), n_new=n_new)
        assert missing.item() == 0
        live = torch.nonzero(n_new)[:, 0]
        cu = torch.zeros(B * K + 1, dtype=torch.int32, device="cuda")
        cu[1:] = torch.cumsum(n_new, 0)
        tokens = best["token"].view(-1)[live].cpu().numpy()
        pos = [positions(n - 1, grid) for n in lens[live].tolist()]
        logits = torch.zeros(B * K, V, device="cuda")
        if len(tokens):
            logits[live] = model(tokens, pos, table, lens, cu, B * K)[:len(tokens)]
        logits = logits.view(B, K, V)
        # every page is held as often as the tables say
        t, n = table.cpu().numpy(), lens.tolist()
        held = np.zeros(n_pages, int)
        for row, m in zip(t, n):
            np.add.at(held, row[:-(-m // P)], 1)
        assert np.array_equal(held, ref.cpu().numpy())
    assert any(d for h in hyp for _, _, d in h)  # a beam has ended on the way
    _, lens, ref, _ = lib.pages_fork(kp, vp, table, lens, ref, ints([-1]))
    assert lens.tolist() == [0] and not ref.any()
