"""spider_decode_tree against the oracle, and the operators for drafting over the cache in
a run together: prefill, drafted steps, rules on the logits, acceptance, eviction.

Bars as for spider_decode_step: states and logits within 2e-2 (bf16) / 1e-4 (fp32) of the
oracle relative to the largest entry, cached keys and values 1e-2 / 1e-5; the weights of a
layer within 2e-2 / 1e-4 of the largest.  Tokens of the drafted run equal those of one
token at a time.
"""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import decode as odec
from oracle import drafting as od
from synth import get_workload
from synth.decoder_inputs import layer_weights
from synth.online_inputs import unembed
from gpu_common import log, need_gpu, rel_err

pytestmark = pytest.mark.gpu


def setup(wl, layers, B, cap, seed=0, d_scale=0.5):
    L = need_gpu()
    dec = dataclasses.replace(get_workload(wl).dec, L=layers)
    bf16 = dec.dtype == "bf16"
    cfg = L.decoder_cfg(layers, dec.d, dec.H, dec.d_ff, L.BF16 if bf16 else L.F32, dec.eps, dec.theta)
    W = [layer_weights(dec, l, seed, "cuda") for l in range(layers)]
    kv = L.kv_cache(cfg, B, cap, "cuda")
    return L, dec, bf16, cfg, W, kv


def rows(dec, shape, seed):
    x = torch.randn(*shape, dec.d, generator=torch.Generator().manual_seed(seed)) * 0.5
    return x.to(torch.bfloat16 if dec.dtype == "bf16" else torch.float32)


CASES = {
    "tiny": ("tiny", 2, [30, 0, 17], [40, 0, 17], [[-1, 0, 0, 1, -1], [-1, -1, 1, 2, -2], [-1, 0, 1, -2, -2]]),
    "tiny_chain": ("tiny", 2, [33, 9], None, None),
    "7b_tree": ("llava15_7b", 1, [50, 21], [300, 21], [[-1, 0, 0, 1, 2, 2, -1], [-1, 0, 1, 2, 3, 4, -2]]),
    "7b_one_row": ("llava15_7b", 1, [64], [64], [[-1]]),
}


@pytest.mark.parametrize("case", list(CASES))
def test_decode_tree_matches_the_oracle(case):
    wl, layers, lens, pos, parents = CASES[case]
    B, cap, V = len(lens), max(lens) + 9, 512
    T = len(parents[0]) if parents else 4
    L, dec, bf16, cfg, W, kv = setup(wl, layers, B, cap)
    for i, c in enumerate((kv["k"], kv["v"])):
        c.copy_(torch.randn(c.shape, generator=torch.Generator().manual_seed(7 + i)))
    k0, v0 = (c.double().cpu().numpy() for c in (kv["k"], kv["v"]))
    x = rows(dec, (B, T), 3)
    wu = unembed(dec, V, seed=3)
    fn = torch.rand(dec.d, generator=torch.Generator().manual_seed(5)) + 0.5
    aw = torch.rand(layers, B, dec.H, cap).cuda()
    aw0 = aw.double().cpu().numpy()
    h, logits, nxt = L.decode_tree(cfg, W, lens, x.cuda(), kv, parents=parents, pos=pos, final_norm=fn.cuda(),
                                   w_unembed=wu.cuda(), attn_weights=aw)
    pr = np.array(parents if parents else [list(range(-1, T - 1))] * B)
    wts = lambda l: {k: v.double().numpy() for k, v in layer_weights(dec, l, 0, "cpu").items()}  # noqa: E731
    recipe = "bf16" if bf16 else "f32"
    ho = od.decode_tree(x.double().numpy(), wts, k0, v0, lens, pos or lens, pr, dec, recipe, aw0)
    tol, tol_kv = (2e-2, 1e-2) if bf16 else (1e-4, 1e-5)
    live = pr > -2
    lo = odec.lm_head(ho.reshape(B * T, -1), fn.numpy(), wu.double().numpy(), dec.eps, recipe).reshape(B, T, V)
    hg, lg = h.cpu().numpy()[live], logits.cpu().numpy()[live]
    eh, el = rel_err(hg, ho[live]), rel_err(lg, lo[live])
    ek, ev = rel_err(kv["k"].double().cpu().numpy(), k0), rel_err(kv["v"].double().cpu().numpy(), v0)
    ew = rel_err(aw.double().cpu().numpy(), aw0)
    log(f"[tree] {case}: h {eh:.2e} logits {el:.2e} k {ek:.2e} v {ev:.2e} weights {ew:.2e}")
    assert eh <= tol and el <= tol and ek <= tol_kv and ev <= tol_kv and ew <= tol
    top = np.sort(lo[live], axis=-1)
    sure = top[:, -1] - top[:, -2] > 2 * tol * np.abs(lo[live]).max()
    assert np.array_equal(nxt.cpu().numpy()[live][sure], lo[live].argmax(-1)[sure])
    # slots past the present nodes, and rows of other samples, are as they were
    for b in range(B):
        n = lens[b] + int(live[b].sum())
        assert np.array_equal(kv["k"][:, b, n:].double().cpu().numpy(), k0[:, b, n:])


@pytest.mark.parametrize("wl", ["tiny", "llava15_7b"])
def test_one_node_is_a_decode_step(wl):
    L, dec, bf16, cfg, W, kv = setup(wl, 2, 2, 60)
    for c in (kv["k"], kv["v"]):
        c.copy_(torch.randn(c.shape, generator=torch.Generator().manual_seed(9)))
    kv2 = {"k": kv["k"].clone(), "v": kv["v"].clone()}
    kv2["desc"] = type(kv["desc"])(kv2["k"].data_ptr(), kv2["v"].data_ptr(), 60)
    x = rows(dec, (2, 1), 4).cuda()
    h, _, _ = L.decode_tree(cfg, W, [40, 13], x, kv)
    h2, _, _ = L.decode_step(cfg, W, [40, 13], x[:, 0], kv2)
    tol = 2e-2 if bf16 else 1e-4
    assert rel_err(h[:, 0].cpu().numpy(), h2.cpu().numpy()) <= tol
    assert rel_err(kv["k"].float().cpu().numpy(), kv2["k"].float().cpu().numpy()) <= tol


def accept(nxt, tokens, parents):
    """The nodes on the path of the arg maxes from the root, and the token after them."""
    path, cur = [0], 0
    while True:
        want = int(nxt[cur])
        hit = [t for t in range(cur + 1, len(parents)) if parents[t] == cur and int(tokens[t]) == want]
        if not hit:
            return path, want
        cur = hit[0]
        path.append(cur)


def rules(V, B, rng):
    f = lambda lo, hi: torch.from_numpy(rng.uniform(lo, hi, B).astype(np.float32)).cuda()  # noqa: E731
    ids = torch.from_numpy(np.stack([rng.choice(V, 5, replace=False) for _ in range(B)]).astype(np.int32)).cuda()
    bias = torch.from_numpy(rng.normal(0, 1.0, (B, 5)).astype(np.float32)).cuda()
    allowed = torch.from_numpy(rng.integers(-2**31, 2**31, (V + 31) // 32).astype(np.int32)).cuda()
    return dict(repetition=f(1.0, 1.4), frequency=f(0, 0.3), presence=f(0, 0.3), bias_ids=ids, bias=bias, mask=allowed)


def test_drafting_gives_the_tokens_of_plain_decoding_and_eviction_goes_on():
    B, V, n_new, T, cap, keep = 2, 500, 20, 6, 80, 40
    L, dec, _, cfg, W, kv = setup("tiny", 2, B, cap)
    rng = np.random.default_rng(11)
    emb = torch.randn(V, dec.d, generator=torch.Generator().manual_seed(1)).cuda()
    wu, fn = unembed(dec, V, seed=3).cuda() * 20, torch.ones(dec.d).cuda()
    cu = np.array([0, 31, 45], np.int32)
    prompt = [rng.integers(0, V, cu[b + 1] - cu[b]).astype(np.int32) for b in range(B)]
    x = emb[torch.from_numpy(np.concatenate(prompt)).long().cuda()].contiguous()
    codes = np.zeros((2, 45), np.uint8)
    codes[1, :20] = 1
    rl = rules(V, B, rng)
    history = torch.zeros(B, 200, dtype=torch.int32).cuda()
    n_prompt = torch.tensor([len(p) - 1 for p in prompt], dtype=torch.int32).cuda()

    def start():
        kv["k"].zero_(), kv["v"].zero_()
        L.prefill_kv(cfg, W, cu, x, codes, kv)
        said = [list(p) for p in prompt]   # the last one is not decided yet: its logits come from a step of its own
        # the prompt's last token is run again as the first root, so its slot is given back
        return said, np.array([len(p) - 1 for p in prompt], np.int32)

    def adjust(logits, said, **kw):
        # the history ends before the root, whose token is a node's
        for b in range(B):
            history[b, :len(said[b]) - 1] = torch.tensor(said[b][:-1], dtype=torch.int32)
        n = torch.tensor([len(s) - 1 for s in said], dtype=torch.int32).cuda()
        return L.adjust_logits(logits, history, n, n_prompt=n_prompt, **rl, **kw)[1].cpu().numpy()

    # one token at a time
    said, lens = start()
    for _ in range(n_new):
        last = torch.tensor([s[-1] for s in said]).cuda()
        _, logits, _ = L.decode_step(cfg, W, lens, emb[last].contiguous(), kv, fn, wu)
        tok = adjust(logits.unsqueeze(1), said, node_tokens=last.int().unsqueeze(1).contiguous())
        lens = lens + 1
        for b in range(B):
            said[b].append(int(tok[b, 0]))
    plain = [list(s) for s in said]

    # drafted: a chain of guesses (some wrong) with a wrong sibling
    said, lens = start()
    aw = torch.zeros(2, B, dec.H, cap).cuda()
    steps = 0
    parents = np.array([[-1, 0, 1, 0, 2, 4]] * B, np.int32)
    while min(len(s) - len(p) for s, p in zip(said, prompt)) < n_new:
        steps += 1
        tokens = np.zeros((B, T), np.int32)
        for b in range(B):
            truth = plain[b][len(said[b]):len(said[b]) + 4] + [1, 2, 3, 4]
            tokens[b] = [said[b][-1], truth[0], truth[1], (truth[0] + 1) % V, truth[2], truth[3]]
            if rng.random() < 0.5:
                tokens[b, rng.integers(1, T)] = rng.integers(0, V)
        dt = torch.from_numpy(tokens).cuda()
        mask, _ = L.tree_mask(parents)
        _, logits, _ = L.decode_tree(cfg, W, lens, emb[dt.long()].contiguous(), kv, parents=parents, final_norm=fn,
                                     w_unembed=wu, attn_weights=aw)
        nxt = adjust(logits, said, node_tokens=dt, tree_mask=torch.from_numpy(mask).cuda())
        idx, count = np.zeros((1, B, 1, T), np.int32), np.zeros(B, np.int32)
        for b in range(B):
            path, after = accept(nxt[b], tokens[b], parents[b])
            idx[0, b, 0, :len(path)], count[b] = path, len(path)
            said[b] += [int(t) for t in tokens[b][path[1:]]] + [after]
        L.cache_compact(kv["k"].view(2, B, cap, dec.H, -1), kv["v"].view(2, B, cap, dec.H, -1),
                        torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(),
                        base=torch.from_numpy(lens).cuda(), weights=aw)
        lens = lens + count
        if lens.max() + T > cap:
            break
    for b in range(B):
        m = min(len(said[b]), len(plain[b]))
        assert said[b][:m] == plain[b][:m]
    log(f"[drafting] {steps} steps for {[len(s) - len(p) for s, p in zip(said, prompt)]} tokens")
    assert steps < n_new

    # eviction: each head keeps its own slots, and the next step attends to what is left
    k0, v0, w0 = (t.double().cpu().numpy() for t in (kv["k"], kv["v"], aw))
    k5, v5 = (t.view(2, B, cap, dec.H, -1) for t in (kv["k"], kv["v"]))
    dl = torch.from_numpy(lens).cuda()
    sel, new = L.cache_select(aw, dl, keep, n_first=2, n_last=8)
    L.cache_compact(k5, v5, sel, new, weights=aw)
    ref, rnew = od.cache_select(w0, lens, keep, 2, 8)
    assert np.array_equal(sel.cpu().numpy(), ref) and np.array_equal(new.cpu().numpy(), rnew)
    shape = (2, B, cap, dec.H, dec.d // dec.H)
    k1, v1 = (od.cache_compact(t.reshape(shape), t.reshape(shape), ref, rnew).reshape(t.shape) for t in (k0, v0))
    assert np.array_equal(kv["k"].double().cpu().numpy(), k1) and np.array_equal(kv["v"].double().cpu().numpy(), v1)
    xr = emb[torch.tensor([[s[-1], 3, 4] for s in said]).cuda()].contiguous()
    h, _, _ = L.decode_tree(cfg, W, rnew, xr, kv, parents=[[-1, 0, 0]] * B, pos=lens)
    wts = lambda l: {k: v.double().cpu().numpy() for k, v in W[l].items()}  # noqa: E731
    ho = od.decode_tree(xr.double().cpu().numpy(), wts, k1, v1, rnew, lens, np.array([[-1, 0, 0]] * B), dec, "f32")
    assert rel_err(h.cpu().numpy(), ho) <= 1e-4


def test_refusals():
    L, dec, _, cfg, W, kv = setup("tiny", 2, 2, 20)
    x = rows(dec, (2, 3), 1).cuda()
    bad = [
        lambda: L.decode_tree(cfg, W, [18, 0], x, kv),                       # 3 nodes past 20 slots
        lambda: L.decode_tree(cfg, W, [-1, 0], x, kv),
        lambda: L.decode_tree(cfg, W, [0, 0], x, kv, pos=[-1, 0]),
        lambda: L.decode_tree(cfg, W, [0, 0], x, kv, parents=[[-1, 1, 0]] * 2),
        lambda: L.decode_tree(cfg, W, [0, 0], x, kv, parents=[[-1, 0]] * 2),
        lambda: L.decode_tree(cfg, W, [0, 0, 0], x, kv),
        lambda: L.decode_tree(cfg, W, [0, 0], x[:, :, :64].contiguous(), kv),
        lambda: L.decode_tree(cfg, W, [0, 0], x.bfloat16(), kv),
        lambda: L.decode_tree(cfg, W, [0, 0], x[:1], kv),
        lambda: L.decode_tree(cfg, W, [0, 0], x, kv, attn_weights=torch.zeros(2, 2, 4, 19).cuda()),
        lambda: L.decode_tree(cfg, W, [0, 0], x, kv, w_unembed=torch.zeros(64, dec.d).cuda()),
    ]
    before = kv["k"].clone()
    for f in bad:
        with pytest.raises((ValueError, TypeError, L.SpiderError)):
            f()
    assert torch.equal(kv["k"], before)
