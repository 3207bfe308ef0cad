"""The drafted step that README.md shows, run as it stands: its tokens are those of one token
at a time, and its evictions see the accepted nodes."""
import os
import re

import numpy as np
import pytest
import torch

from synth.online_inputs import unembed
from test_gpu_decode_tree import accept, rules, setup

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_the_drafted_step():
    step = [c for c in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "decode_tree" in c]
    assert len(step) == 1
    code = compile(step[0], "README.md", "exec")
    B, V, T, cap, n_new = 2, 500, 6, 600, 40
    L, dec, _, cfg, W, kv = setup("tiny", 2, B, cap)
    rng = np.random.default_rng(5)
    emb = torch.randn(V, dec.d, generator=torch.Generator().manual_seed(1)).cuda()
    head, norm = unembed(dec, V, seed=3).cuda() * 20, torch.ones(dec.d).cuda()
    sizes = [571, 540]
    prompt = [rng.integers(0, V, n).astype(np.int32) for n in sizes]
    rl = rules(V, B, rng)
    history = torch.zeros(B, 800, dtype=torch.int32).cuda()
    n_prompt = torch.tensor([n - 1 for n in sizes], dtype=torch.int32).cuda()
    base = np.array(sizes, np.int32) - 1   # the prompt's last token is the first root

    def start():
        cu = np.array([0, sizes[0], sum(sizes)], np.int32)
        L.prefill_kv(cfg, W, cu, emb[torch.from_numpy(np.concatenate(prompt)).long().cuda()].contiguous(),
                     np.zeros((2, sum(sizes)), np.uint8), kv)
        return [list(p) for p in prompt]

    def past(said):  # before the root, whose token is a node's
        for b in range(B):
            history[b, :len(said[b]) - 1] = torch.tensor(said[b][:-1], dtype=torch.int32)
        return torch.tensor([len(s) - 1 for s in said], dtype=torch.int32).cuda()

    said, lens = start(), base.copy()
    for _ in range(n_new):
        if lens.max() == cap:
            break
        last = torch.tensor([s[-1] for s in said]).cuda()
        _, logits, _ = L.decode_step(cfg, W, lens, emb[last].contiguous(), kv, norm, head)
        n = past(said)
        tok = L.adjust_logits(logits.unsqueeze(1), history, n, n_prompt=n_prompt, node_tokens=last.int().unsqueeze(1), **rl)[1]
        lens = lens + 1
        for b in range(B):
            said[b].append(int(tok[b, 0]))
    plain = said

    said = start()
    evictions = []

    def select(weights, lens, keep, **kw):
        chosen = L.cache_select(weights, lens, keep, **kw)
        evictions.append((lens.cpu().numpy(), kv["k"].clone(), chosen[0].clone()))
        return chosen

    def verify(following, tokens, parents):
        nxt, tokens = following.cpu().numpy(), tokens.cpu().numpy()
        accepted, count = np.zeros((1, B, 1, T), np.int32), np.zeros(B, np.int32)
        for b in range(B):
            path, after = accept(nxt[b], tokens[b], parents[b])
            accepted[0, b, 0, :len(path)], count[b] = path, len(path)
            said[b] += [int(t) for t in tokens[b][path[1:]]] + [after]
        return accepted, count

    parents = np.array([[-1, 0, 1, 0, 2, 4]] * B, np.int32)
    names = dict(cfg=cfg, W=W, lens=base.copy(), pos=base.copy(), kv=kv, parents=parents, norm=norm, head=head, history=history,
                 rep=rl["repetition"], ids=rl["bias_ids"], bias=rl["bias"], grammar=rl["mask"], torch=torch, T=T, cap=cap,
                 weights=torch.zeros(2, B, dec.H, cap).cuda(), k=kv["k"].view(2, B, cap, dec.H, -1),
                 v=kv["v"].view(2, B, cap, dec.H, -1), verify=verify, tree_mask=L.tree_mask, decode_tree=L.decode_tree,
                 cache_compact=L.cache_compact, cache_select=select)
    # the README's rules: repetition, biases and a grammar, no frequency and presence penalties, all of the history said
    names["adjust_logits"] = lambda *a, **kw: L.adjust_logits(*a, n_prompt=n_prompt, frequency=rl["frequency"], presence=rl["presence"], **kw)
    while len(evictions) < 2:  # every step says a token at least
        tokens = np.zeros((B, T), np.int32)
        for b in range(B):
            truth = plain[b][len(said[b]):len(said[b]) + 4] + [1, 2, 3, 4]
            tokens[b] = [said[b][-1], truth[0], truth[1], (truth[0] + 1) % V, truth[2], truth[3]]
        before, done, pos = [len(s) for s in said], len(evictions), names["pos"].copy()
        names.update(tokens=torch.from_numpy(tokens).cuda(), x=emb[torch.from_numpy(tokens).long().cuda()].contiguous(), n_history=past(said))
        lens = names["lens"].copy()
        exec(code, names)
        grown = lens + [len(s) - n for s, n in zip(said, before)]
        assert np.array_equal(names["pos"], pos + grown - lens)
        if len(evictions) == done:
            assert np.array_equal(names["lens"], grown)
            if done == 0:
                for b in range(B):
                    m = min(len(said[b]), len(plain[b]))
                    assert said[b][:m] == plain[b][:m]
            continue
        seen, k, idx = evictions[-1]
        assert np.array_equal(seen, grown) and np.array_equal(names["lens"], np.minimum(grown, 512))
        for b in range(B):
            assert idx[:, b, :, -64:].cpu().tolist() == [[list(range(grown[b] - 64, grown[b]))] * dec.H] * 2
        want = torch.gather(k.view(2, B, cap, dec.H, -1), 2, idx.long().transpose(2, 3)[..., None].expand(-1, -1, -1, -1, dec.d // dec.H))
        assert torch.equal(names["k"][:, :, :512], want)
