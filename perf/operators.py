"""Performance cases of the operators for drafting over the pruned cache: what a serving loop calls around the decoder.

  tree    attention of a tree of drafted tokens over a key/value cache (spider_tree_attention); one token per sample is
          its smallest tree; with ``weights`` it also adds up the attention weight that every cached slot receives
  evict   the slots of a cache that its accumulated attention weight keeps (spider_cache_select), and their keys, values
          and weights moved into a smaller cache (spider_cache_compact)
  adjust  penalties for repeated tokens, biases and grammar masks on logits, and the arg max (spider_adjust_logits), for
          one row per sample or for the nodes of a tree

Head layouts and widths are those of the repository's decoders (32 or 40 heads of 128; heads of 64 and 32 in fp32) and
of grouped heads; lengths are pruned prompts (200, 705, 2944 slots) and longer caches; the vocabulary is the repository's
32000 and larger ones.  ``exact`` evaluates the same definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"


def listed():
    return [
        # one sample's next token over a pruned prompt of the LLaVA-1.5-7B shape: launches and latency
        dict(name="tree_1_of_200", kind="tree", B=1, T=1, H=32, Hkv=32, dh=128, len=200, dtype="bf16", weights=False, heads_first=False),
        # sixteen drafted tokens over a five-tile prompt, the weights kept for a later eviction
        dict(name="tree_16_of_705", kind="tree", B=1, T=16, H=32, Hkv=32, dh=128, len=705, dtype="bf16", weights=True, heads_first=False),
        # a fp32 decoder of 8 heads of 64 at two samples
        dict(name="tree_13_f32", kind="tree", B=2, T=13, H=8, Hkv=8, dh=64, len=1500, dtype="f32", weights=True, heads_first=False),
        # a batch of eight with large trees over long caches of grouped heads
        dict(name="tree_61_grouped", kind="tree", B=8, T=61, H=32, Hkv=8, dh=128, len=16384, dtype="bf16", weights=False, heads_first=True),
        # plain decoding of sixteen samples over long caches of grouped heads, the weights kept
        dict(name="tree_1_of_32768", kind="tree", B=16, T=1, H=32, Hkv=8, dh=128, len=32768, dtype="bf16", weights=True, heads_first=False),
        # a small fp32 cache, the same tokens kept for all heads
        dict(name="evict_small_f32", kind="evict", L=2, B=3, Hkv=4, dh=32, len=333, keep=100, first=4, last=32, dtype="f32", shared=True, heads_first=False),
        # every layer of a 7B cache after an unpruned prompt: 2944 slots down to 576, each head its own
        dict(name="evict_7b_2944", kind="evict", L=32, B=1, Hkv=32, dh=128, len=2944, keep=576, first=4, last=64, dtype="bf16", shared=False, heads_first=False),
        # long ragged caches of grouped heads, a quarter kept
        dict(name="evict_65536", kind="evict", L=4, B=2, Hkv=8, dh=128, len=65536, keep=16384, first=4, last=1024, dtype="bf16", shared=False, heads_first=True),
        # one sample's logits before its next token is chosen
        dict(name="adjust_1", kind="adjust", B=1, T=1, V=32000, history=700, prompt=600, bias=8, mask=True, dtype="f32"),
        # the logits of 32 tree nodes for each of eight samples, under a grammar
        dict(name="adjust_tree_8x31", kind="adjust", B=8, T=31, V=32000, history=2900, prompt=2000, bias=100, mask=True, dtype="f32"),
        # a batch of 64 over a large vocabulary, bf16 logits, long histories
        dict(name="adjust_64_wide", kind="adjust", B=64, T=1, V=151000, history=12000, prompt=8000, bias=300, mask=False, dtype="bf16"),
    ]


HEADS = ((32, 32, 128), (32, 32, 128), (40, 40, 128), (32, 8, 128), (32, 8, 128), (16, 4, 64), (12, 12, 64), (16, 16, 80), (8, 1, 256))
HEADS_F32 = ((8, 8, 64), (4, 4, 32), (8, 2, 128), (6, 2, 48))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(("tree", "tree", "tree", "evict", "adjust"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if kind == "tree":
        H, Hkv, dh = rng.choice(HEADS if dtype == "bf16" else HEADS_F32)
        return dict(kind=kind, B=_log_int(rng, 1, 32), T=rng.choice((1, 1, _log_int(rng, 2, 128), _log_int(rng, 2, 128))), H=H, Hkv=Hkv, dh=dh,
                    len=_log_int(rng, 1, 40000), dtype=dtype, weights=rng.random() < 0.4, heads_first=rng.random() < 0.4)
    if kind == "evict":
        _, Hkv, dh = rng.choice(HEADS if dtype == "bf16" else HEADS_F32)
        n = _log_int(rng, 16, 80000)
        keep = max(2, min(n, int(n * rng.uniform(0.02, 0.9))))
        first = rng.randint(0, min(8, keep // 2))
        return dict(kind=kind, L=_log_int(rng, 1, 40), B=_log_int(rng, 1, 8), Hkv=Hkv, dh=dh, len=n, keep=keep, first=first,
                    last=rng.randint(0, (keep - first) // 2), dtype=dtype, shared=rng.random() < 0.4, heads_first=rng.random() < 0.4)
    history = _log_int(rng, 1, 20000)
    return dict(kind=kind, B=_log_int(rng, 1, 96), T=rng.choice((1, 1, _log_int(rng, 2, 64))), V=rng.choice((32000, 32064, _log_int(rng, 500, 160000))),
                history=history, prompt=rng.randint(0, history), bias=rng.choice((0, _log_int(rng, 1, 400))), mask=rng.random() < 0.5, dtype=dtype)


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = (max(most.get(c["kind"], (0, 0))[0], w["bytes"]), max(most.get(c["kind"], (0, 0))[1], w["flops"]))
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["bytes"] <= most[c["kind"]][0] and w["flops"] <= most[c["kind"]][1]:
            return c


# -------------------------------------------------------------------------------------------------------------- shapes
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _size(name):
    return 2 if name == "bf16" else 4


def _lens(c):
    """Filled slots of each sample: prompts differ in length, and the longest comes first."""
    return [c["len"] - (b * 37) % (c["len"] // 3 + 1) for b in range(c["B"])]


def _nodes(c):
    """Live nodes of each sample's tree: some drafts end early."""
    return [c["T"] - (b % 3 if c["T"] > 3 else 0) for b in range(c["B"])]


def work(c):
    es = _size(c["dtype"])
    if c["kind"] == "tree":
        lens, nodes = _lens(c), _nodes(c)
        slots = sum(n + t for n, t in zip(lens, nodes))
        pairs = sum(t * (n + (t + 1) / 2) for n, t in zip(lens, nodes)) * c["H"]
        byts = 2 * slots * c["Hkv"] * c["dh"] * es + 2 * sum(nodes) * c["H"] * c["dh"] * es + c["B"] * c["T"] * (8 * ((c["T"] + 63) // 64))
        if c["weights"]:
            byts += (sum(lens) + slots) * c["Hkv"] * 4
        return {"bytes": float(byts), "flops": 4.0 * pairs * c["dh"]}
    if c["kind"] == "evict":
        lens = _lens(c)
        groups = 1 if c["shared"] else c["Hkv"]
        kept = sum(min(c["keep"], n) for n in lens)
        byts = c["L"] * (sum(lens) * c["Hkv"] * 4 + c["B"] * groups * c["keep"] * 4 + 2 * kept * c["Hkv"] * (2 * c["dh"] * es + 4))
        return {"bytes": float(byts), "flops": 0.0}
    rows = sum(_nodes(c))
    byts = rows * c["V"] * (es + 4) + rows * 4 + c["B"] * c["history"] * 4 + c["B"] * c["bias"] * 8
    if c["mask"]:
        byts += rows * ((c["V"] + 31) // 32) * 4
    return {"bytes": float(byts), "flops": 6.0 * rows * c["V"]}


# -------------------------------------------------------------------------------------------------------------- inputs
def _trees(c, rng):
    """Random trees of drafted tokens: every node's parent is an earlier one, or the context (-1); bit u of a node's mask
    is set for its ancestors and itself."""
    B, T = c["B"], c["T"]
    W = (T + 63) // 64
    see = np.zeros((B, T, T), bool)
    for b in range(B):
        parents = np.maximum(-1, np.arange(T) - 1 - rng.integers(0, 1 + np.arange(T) // 2 + 1))
        for t in range(T):
            if parents[t] >= 0:
                see[b, t] = see[b, parents[t]]
            see[b, t, t] = True
    bits = np.zeros((B, T, W * 64), np.uint8)
    bits[:, :, :T] = see
    words = np.packbits(bits, axis=2, bitorder="little").view(np.int64).reshape(B, T, W)
    return torch.from_numpy(words).to(DEV)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _cache(c, cap, lead, gen, fill=True):
    """A cache of [.., cap, Hkv, dh], its slots in the order of tokens or of heads."""
    shape = lead + ((c["Hkv"], cap, c["dh"]) if c["heads_first"] else (cap, c["Hkv"], c["dh"]))
    t = torch.empty(shape, dtype=_dtype(c["dtype"]), device=DEV)
    t.normal_(generator=gen) if fill else t.zero_()
    return t.transpose(-3, -2) if c["heads_first"] else t


def prepare(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    B = c["B"]
    s = {"c": c}
    if c["kind"] == "tree":
        T, H, Hkv, dh = c["T"], c["H"], c["Hkv"], c["dh"]
        cap = (c["len"] + T + 127) // 64 * 64
        s["q"] = (1.5 * torch.randn(B, T, H, dh, generator=gen, device=DEV)).to(_dtype(c["dtype"]))
        s["k"], s["v"] = (_cache(c, cap, (B,), gen) for _ in range(2))
        s["lens"], s["nodes"], s["tree"] = _ints(_lens(c)), _ints(_nodes(c)), _trees(c, rng)
        s["out"] = torch.zeros_like(s["q"])
        if c["weights"]:
            s["w_in"] = torch.rand(B, Hkv, cap, generator=gen, device=DEV)
            s["w_out"] = torch.zeros_like(s["w_in"])
    elif c["kind"] == "evict":
        L, Hkv, keep = c["L"], c["Hkv"], c["keep"]
        cap = (c["len"] + 63) // 64 * 64
        s["k"], s["v"] = (_cache(c, cap, (L, B), gen) for _ in range(2))
        s["lens"] = _ints(_lens(c))
        # accumulated weights: a heavy tail, and slots that never got any
        w = torch.empty(L, B, Hkv, cap, device=DEV).exponential_(generator=gen).pow_(3)
        s["w"] = torch.where(w < 1e-3, torch.zeros_like(w), w)
        s["k_to"], s["v_to"] = (_cache(c, keep, (L, B), gen, fill=False) for _ in range(2))
        s["w_to"] = torch.zeros(L, B, Hkv, keep, device=DEV)
    else:
        T, V = c["T"], c["V"]
        s["logits"] = (2.5 * torch.randn(B, T, V, generator=gen, device=DEV)).to(_dtype(c["dtype"]))
        tokens = np.minimum(rng.zipf(1.3, (B, c["history"] + T)) - 1, V - 1).astype(np.int32)  # few tokens fill most of a text
        s["history"] = torch.from_numpy(np.ascontiguousarray(tokens[:, :c["history"]])).to(DEV)
        s["drafted"] = torch.from_numpy(np.ascontiguousarray(tokens[:, c["history"]:])).to(DEV)
        s["n_history"] = _ints([c["history"] - (b * 37) % (c["history"] // 3 + 1) for b in range(B)])
        s["n_prompt"] = _ints([min(c["prompt"], n) for n in s["n_history"].tolist()])
        s["nodes"], s["tree"] = _ints(_nodes(c)), _trees(c, rng)
        s["rep"], s["freq"], s["pres"] = (torch.from_numpy(rng.uniform(lo, hi, B).astype(np.float32)).to(DEV) for lo, hi in ((1.0, 1.3), (0.0, 0.5), (0.0, 0.8)))
        s["bias_ids"] = s["bias"] = s["mask"] = None
        if c["bias"]:
            ids = np.stack([rng.choice(V, min(V, c["bias"]), replace=False) for _ in range(B)]).astype(np.int32)
            s["bias_ids"] = torch.from_numpy(ids).to(DEV)
            s["bias"] = torch.from_numpy(rng.normal(0, 4, ids.shape).astype(np.float32)).to(DEV)
        if c["mask"]:
            s["mask"] = torch.from_numpy(rng.integers(-2**31, 2**31, (B, T, (V + 31) // 32)).astype(np.int32)).to(DEV)
        s["out"] = torch.zeros(B, T, V, device=DEV)
        s["next"] = torch.full((B, T), -1, dtype=torch.int32, device=DEV)
    return s


# --------------------------------------------------------------------------------------------------------- plain forms
def _sees(s):
    """[B, T, T]: node t sees node u, both alive."""
    B, T, W = s["tree"].shape
    u = torch.arange(T, device=DEV)
    bit = (s["tree"][:, :, u // 64] >> (u % 64)) & 1
    alive = u[None, :] < s["nodes"][:, None]
    return (bit != 0) & alive[:, :, None] & alive[:, None, :]


def _plain_tree(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    B, T, H, dh = q.shape
    cap, Hkv = k.shape[1], k.shape[2]
    G = H // Hkv
    slot = torch.arange(cap, device=DEV)
    node = slot[None] - s["lens"][:, None]
    alive = torch.arange(T, device=DEV)[None] < s["nodes"][:, None]
    in_tree = torch.gather(_sees(s), 2, node.clamp(0, T - 1)[:, None, :].expand(B, T, cap))
    sees = (node < 0)[:, None, :] | (in_tree & (node >= 0)[:, None, :] & (node < T)[:, None, :])
    sees = (sees & alive[:, :, None])[:, None, :, None, :]                              # [B, 1, T, 1, cap]
    rows = q.view(B, T, Hkv, G, dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, dh)
    x = torch.matmul(rows, k.permute(0, 2, 3, 1).contiguous()).view(B, Hkv, T, G, cap) * dh ** -0.5
    x = x.masked_fill(~sees, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(B, Hkv, T * G, cap), v.permute(0, 2, 1, 3).contiguous())
    o = o.view(B, Hkv, T, G, dh).permute(0, 2, 1, 3, 4).reshape(B, T, H, dh).to(s["q"].dtype)
    o = torch.where(alive[:, :, None, None], o, s["out"])
    if not s["c"]["weights"]:
        return {"out": o}
    held = (node < 0)[:, None, :]
    w = torch.where(held, s["w_in"], torch.zeros_like(s["w_in"])) + p.sum((2, 3))
    return {"out": o, "weights": torch.where((node < s["nodes"][:, None])[:, None, :], w, s["w_out"])}


def _plain_evict(s):
    c, w, lens = s["c"], s["w"], s["lens"]
    cap, keep = w.shape[3], c["keep"]
    if c["shared"]:
        w = w.double().sum(2, keepdim=True).float()
    slot = torch.arange(cap, device=DEV)
    n = lens[None, :, None, None]
    always = (slot < c["first"]) | (slot >= n - c["last"])
    key = w.masked_fill(always, math.inf).masked_fill(slot >= n, -math.inf)
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    best = torch.sort(best.masked_fill(best >= n, cap), dim=-1).values
    fills = best < cap
    idx = torch.where(fills, best, -torch.ones_like(best)).int()
    at = torch.where(fills, best, torch.zeros_like(best)).expand(-1, -1, c["Hkv"], -1)  # [L, B, Hkv, keep]
    fills = fills.expand(-1, -1, c["Hkv"], -1)
    moved = [torch.where(fills.transpose(2, 3)[..., None], torch.gather(x, 2, at.transpose(2, 3)[..., None].expand(-1, -1, -1, -1, c["dh"])), y)
             for x, y in ((s["k"], s["k_to"]), (s["v"], s["v_to"]))]
    return {"idx": idx, "lens": torch.clamp(lens, max=keep), "k": moved[0], "v": moved[1],
            "weights": torch.where(fills, torch.gather(s["w"], 3, at), s["w_to"])}


def _plain_adjust(s):
    B, T, V = s["logits"].shape
    n = s["history"].shape[1]
    x = s["logits"].float()
    place = torch.arange(n, device=DEV)[None]
    past = (place < s["n_history"][:, None]).int()
    said = past * (place >= s["n_prompt"][:, None])
    ids = s["history"].long()
    seen = torch.zeros(B, V, dtype=torch.int32, device=DEV).scatter_add_(1, ids, past)
    count = torch.zeros(B, V, dtype=torch.int32, device=DEV).scatter_add_(1, ids, said)
    drafts = torch.zeros(B, T, V, dtype=torch.int32, device=DEV).scatter_add_(2, s["drafted"].long()[:, None].expand(B, T, T), _sees(s).int())
    if T == 1:
        drafts.zero_()  # a single row has no drafted tokens before it
    count = count[:, None] + drafts
    seen = (seen[:, None] + drafts) > 0
    rep, freq, pres = (s[k][:, None, None] for k in ("rep", "freq", "pres"))
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = torch.where(count > 0, x - freq * count.float() - pres, x)
    if s["bias"] is not None:
        x = x + torch.zeros(B, V, device=DEV).scatter_add_(1, s["bias_ids"].long(), s["bias"])[:, None]
    if s["mask"] is not None:
        v = torch.arange(V, device=DEV)
        x = x.masked_fill(((s["mask"][:, :, v // 32] >> (v % 32)) & 1) == 0, -math.inf)
    top = x.amax(-1, keepdim=True)
    first = torch.where(x == top, torch.arange(V, device=DEV, dtype=torch.int32), V).amin(-1).int()
    first = torch.where(top[..., 0] == -math.inf, -torch.ones_like(first), first)
    alive = torch.arange(T, device=DEV)[None] < s["nodes"][:, None]
    return {"logits": torch.where(alive[..., None], x, s["out"]), "next": torch.where(alive, first, s["next"])}


# ------------------------------------------------------------------------------------------------------------ one pass
def run(s):
    kind = s["c"]["kind"]
    if not own:
        return {"tree": _plain_tree, "evict": _plain_evict, "adjust": _plain_adjust}[kind](s)
    from paper_2609_34977_amd import _lib
    if kind == "tree":
        weights = dict(weights_in=s["w_in"], weights_out=s["w_out"]) if s["c"]["weights"] else {}
        out = _lib.tree_attention(s["q"], s["k"], s["v"], s["lens"], n_nodes=s["nodes"], tree_mask=s["tree"], out=s["out"], **weights)
        return {"out": out, "weights": s["w_out"]} if weights else {"out": out}
    if kind == "evict":
        c = s["c"]
        idx, lens = _lib.cache_select(s["w"], s["lens"], c["keep"], n_first=c["first"], n_last=c["last"], shared=c["shared"])
        _lib.cache_compact(s["k"], s["v"], idx, lens, k_out=s["k_to"], v_out=s["v_to"], weights=s["w"], weights_out=s["w_to"])
        return {"idx": idx, "lens": lens, "k": s["k_to"], "v": s["v_to"], "weights": s["w_to"]}
    drafted = dict(node_tokens=s["drafted"], tree_mask=s["tree"]) if s["c"]["T"] > 1 else {}
    logits, following = _lib.adjust_logits(s["logits"], s["history"], s["n_history"], n_prompt=s["n_prompt"], n_nodes=s["nodes"], repetition=s["rep"],
                                           frequency=s["freq"], presence=s["pres"], bias_ids=s["bias_ids"], bias=s["bias"], mask=s["mask"],
                                           out=s["out"], next_ids=s["next"], **drafted)
    return {"logits": logits, "next": following}


# ------------------------------------------------------------------------------------------------------------- 64 bits
def _exact_tree(s):
    c = s["c"]
    G = c["H"] // c["Hkv"]
    q = s["q"].double()
    out = s["out"].double().clone()
    w_out = s["w_out"].double().clone() if c["weights"] else None
    words = s["tree"].cpu().numpy().view(np.uint64)
    for b, (n, t) in enumerate(zip(_lens(c), _nodes(c))):
        sees = np.ones((t, n + t), bool)
        for i in range(t):
            sees[i, n:] = [bool(words[b, i, u // 64] >> np.uint64(u % 64) & np.uint64(1)) for u in range(t)]
        hidden = torch.from_numpy(~sees).to(DEV)
        for h in range(c["Hkv"]):
            K, V = s["k"][b, :n + t, h].double(), s["v"][b, :n + t, h].double()
            x = torch.einsum("tgd,nd->tgn", q[b, :t, h * G:(h + 1) * G], K) / math.sqrt(c["dh"])
            p = torch.softmax(x.masked_fill(hidden[:, None], -math.inf), -1)
            out[b, :t, h * G:(h + 1) * G] = torch.einsum("tgn,nd->tgd", p, V)
            if c["weights"]:
                w_out[b, h, :n + t] = p.sum((0, 1))
                w_out[b, h, :n] += s["w_in"][b, h, :n].double()
    return {"out": out, "weights": w_out} if c["weights"] else {"out": out}


def _exact_evict(s):
    c = s["c"]
    w = s["w"].cpu().numpy().astype(np.float64)
    moved = {x: s[x + "_to"].double().clone() for x in ("k", "v", "w")}
    for layer in range(c["L"]):
        for b, n in enumerate(_lens(c)):
            total = w[layer, b, :, :n].sum(0).astype(np.float32)
            for h in range(c["Hkv"]):
                score = (total if c["shared"] else w[layer, b, h, :n]).astype(np.float64)
                score[:c["first"]] = math.inf
                score[max(0, n - c["last"]):] = math.inf
                kept = np.sort(np.argsort(-score, kind="stable")[:c["keep"]])
                at = torch.from_numpy(kept).to(DEV)
                moved["k"][layer, b, :len(kept), h] = s["k"][layer, b, at, h].double()
                moved["v"][layer, b, :len(kept), h] = s["v"][layer, b, at, h].double()
                moved["w"][layer, b, h, :len(kept)] = s["w"][layer, b, h, at].double()
    return {"idx": None, "lens": None, "k": moved["k"], "v": moved["v"], "weights": moved["w"]}


def _exact_adjust(s):
    c = s["c"]
    x = s["logits"].double().cpu().numpy()
    out = s["out"].double().cpu().numpy()
    history, drafted, words = s["history"].cpu().numpy(), s["drafted"].cpu().numpy(), s["tree"].cpu().numpy().view(np.uint64)
    rep, freq, pres = (s[k].cpu().numpy().astype(np.float64) for k in ("rep", "freq", "pres"))
    for b, t in enumerate(_nodes(c)):
        n, n_prompt = int(s["n_history"][b]), int(s["n_prompt"][b])
        for i in range(t):
            path = [drafted[b, u] for u in range(t) if words[b, i, u // 64] >> np.uint64(u % 64) & np.uint64(1)] if c["T"] > 1 else []
            said = np.bincount(np.concatenate([history[b, n_prompt:n], np.array(path, np.int32)]).astype(np.int64), minlength=c["V"])
            seen = (np.bincount(history[b, :n_prompt], minlength=c["V"]) + said) > 0
            y = x[b, i].copy()
            y[seen] = np.where(y[seen] > 0, y[seen] / rep[b], y[seen] * rep[b])
            y -= freq[b] * said + pres[b] * (said > 0)
            if s["bias"] is not None:
                np.add.at(y, s["bias_ids"][b].cpu().numpy(), s["bias"][b].cpu().numpy().astype(np.float64))
            if s["mask"] is not None:
                allowed = np.unpackbits(s["mask"][b, i].cpu().numpy().view(np.uint8), bitorder="little")[:c["V"]]
                y[allowed == 0] = -math.inf
            out[b, i] = y
    return {"logits": torch.from_numpy(out), "next": None}


def exact(c, seed):
    if c["kind"] == "adjust" and c["B"] * c["T"] * c["V"] > 4e7:
        return None
    if c["kind"] == "evict" and c["L"] * c["B"] * c["Hkv"] * c["len"] > 2e7:
        return None
    return {"tree": _exact_tree, "evict": _exact_evict, "adjust": _exact_adjust}[c["kind"]](prepare(c, seed))
