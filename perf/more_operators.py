"""Performance cases of the operators for beams and chunks over a paged cache: what a serving loop calls around the decoder
when sequences share pages.

  rope    rotary positions with several axes (time, height, width) on queries and keys, the keys and values of the new
          tokens stored in their pages (spider_rope_append)
  attn    attention of a chunk of new tokens per sequence over the pages (spider_paged_attention); one new token per
          sequence is its smallest chunk
  fork    the next step's page tables: sequences continued by several beams, by one or by none, last pages copied before
          two of them write, room for the new tokens (spider_pages_fork)
  beam    beam search's choice over beams and vocabulary, and the token histories that follow it (spider_beam_select)

Head layouts and widths are those of the repository's decoders (32 or 40 heads of 128; heads of 64 and 32 in fp32) and of
grouped heads; lengths are pruned prompts (200, 705, 2944 slots) and longer caches; the vocabulary is the repository's
32000 and larger ones.  ``exact`` evaluates the same definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
PATCHES, SIDE = 576, 24  # an image tile of 24 x 24 patches


def listed():
    return [
        # one sample's next token: launches and latency
        dict(name="rope_1", kind="rope", B=1, new=1, mixed=False, len=705, H=32, Hkv=32, dh=128, rot=128, axes=3, inter=False, page=16, at=705, dtype="bf16", heads_first=False),
        # a fp32 decoder with partly rotated heads, far positions
        dict(name="rope_f32_far", kind="rope", B=5, new=77, mixed=False, len=1500, H=6, Hkv=2, dh=48, rot=40, axes=3, inter=True, page=32, at=900000, dtype="f32", heads_first=True),
        # the prompts of eight samples of five image tiles each, in one packed batch
        dict(name="rope_8x2944", kind="rope", B=8, new=2944, mixed=False, len=2944, H=32, Hkv=8, dh=128, rot=128, axes=3, inter=True, page=64, at=0, dtype="bf16", heads_first=False),
        # one sample's next token over a pruned prompt: launches and latency
        dict(name="attn_1_of_200", kind="attn", B=1, new=1, mixed=False, len=200, H=32, Hkv=32, dh=128, window=0, page=16, dtype="bf16", heads_first=False),
        # a fp32 decoder of grouped heads, chunks that end early, a window
        dict(name="attn_f32_window", kind="attn", B=3, new=70, mixed=False, len=1500, H=6, Hkv=2, dh=48, window=300, page=16, dtype="f32", heads_first=False),
        # plain decoding of sixteen samples over long caches of grouped heads
        dict(name="attn_1_of_32768", kind="attn", B=16, new=1, mixed=False, len=32768, H=32, Hkv=8, dh=128, window=0, page=64, dtype="bf16", heads_first=False),
        # one prompt's next chunk among fifteen sequences that decode
        dict(name="attn_mixed_705", kind="attn", B=16, new=705, mixed=True, len=8192, H=32, Hkv=8, dh=128, window=0, page=32, dtype="bf16", heads_first=True),
        # a chunk of a long prompt
        dict(name="attn_4096_of_32768", kind="attn", B=1, new=4096, mixed=False, len=32768, H=32, Hkv=8, dh=128, window=0, page=128, dtype="bf16", heads_first=False),
        # four beams of one sample
        dict(name="fork_4_f32", kind="fork", groups=1, beams=4, L=2, prompt=100, len=133, n_new=1, Hkv=4, dh=32, page=16, dtype="f32", heads_first=False),
        # eight samples of four beams over the prompts of the LLaVA-1.5-7B shape, all layers
        dict(name="fork_8x4_705", kind="fork", groups=8, beams=4, L=32, prompt=640, len=705, n_new=1, Hkv=32, dh=128, page=16, dtype="bf16", heads_first=False),
        # one sample's four beams before the next token
        dict(name="beam_4", kind="beam", B=1, K=4, M=4, V=32000, history=705, eos=2, done=False, dtype="f32"),
        # 64 samples of eight beams over a large vocabulary, bf16 logits, some beams finished
        dict(name="beam_64x8_wide", kind="beam", B=64, K=8, M=8, V=151000, history=2000, eos=7, done=True, dtype="bf16"),
    ]


HEADS = ((32, 32, 128), (32, 32, 128), (40, 40, 128), (32, 8, 128), (32, 8, 128), (16, 4, 64), (12, 12, 64), (16, 16, 80), (8, 1, 256))
HEADS_F32 = ((8, 8, 64), (4, 4, 32), (8, 2, 128), (6, 2, 48))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(("rope", "attn", "attn", "fork", "beam"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if kind == "beam":
        K = rng.choice((1, _log_int(rng, 2, 32), _log_int(rng, 2, 32)))
        eos = rng.choice((-1, 2, 7))
        return dict(kind=kind, B=_log_int(rng, 1, 96), K=K, M=_log_int(rng, 2, 32) if K == 1 else K, V=rng.choice((32000, 32064, _log_int(rng, 500, 160000))),
                    history=_log_int(rng, 1, 8000), eos=eos, done=K > 1 and eos >= 0 and rng.random() < 0.7, dtype=dtype)
    H, Hkv, dh = rng.choice(HEADS if dtype == "bf16" else HEADS_F32)
    common = dict(Hkv=Hkv, dh=dh, page=rng.choice((8, 16, 16, 32, 64, 128, 256)), dtype=dtype, heads_first=rng.random() < 0.4)
    if kind == "fork":
        prompt = _log_int(rng, 1, 20000)
        return dict(kind=kind, groups=_log_int(rng, 1, 32), beams=_log_int(rng, 1, 16), L=_log_int(rng, 1, 40), prompt=prompt, len=prompt + _log_int(rng, 1, 500),
                    n_new=rng.choice((0, 1, 1, _log_int(rng, 2, 300))), **common)
    B = _log_int(rng, 1, 32)
    new = rng.choice((1, _log_int(rng, 2, 5000), _log_int(rng, 2, 5000)))
    c = dict(kind=kind, B=B, new=new, mixed=new > 1 and rng.random() < 0.3, len=max(new, _log_int(rng, 1, 40000)), H=H, **common)
    if kind == "attn":
        return dict(c, window=rng.choice((0, 0, _log_int(rng, 1, 8000))))
    rot = rng.choice((dh, dh, dh // 8 * 4 + dh % 8))
    return dict(c, rot=rot, axes=rng.randint(1, min(4, rot // 2)), inter=rng.random() < 0.5, at=rng.choice((0, _log_int(rng, 1, 1000000))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = (max(most.get(c["kind"], (0, 0))[0], w["bytes"]), max(most.get(c["kind"], (0, 0))[1], w["flops"]))
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["bytes"] <= most[c["kind"]][0] and w["flops"] <= most[c["kind"]][1] and _pool(c) <= 4e9:
            return c


# -------------------------------------------------------------------------------------------------------------- shapes
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _size(name):
    return 2 if name == "bf16" else 4


def _news(c):
    """New tokens of each sequence: chunks that end early, or one chunk among sequences that decode."""
    if c["mixed"]:
        return [c["new"]] + [1] * (c["B"] - 1)
    return [c["new"] - (b * 13) % (c["new"] // 3 + 1) for b in range(c["B"])]


def _lens(c):
    """Filled slots of each sequence with its new tokens: prompts differ in length, and the longest comes first."""
    return [max(n, c["len"] - (b * 37) % (c["len"] // 3 + 1)) for b, n in enumerate(_news(c))]


def _fork_lens(c):
    """Filled slots of each beam: a sample's beams share its prompt and are equally long."""
    return [c["len"] - (g * 3) % (c["len"] - c["prompt"] + 1) for g in range(c["groups"]) for _ in range(c["beams"])]


def _parents(c):
    """The beams that the next ones continue: two take the first one, the others the next ones, so that the last ends;
    every fifth sample has ended altogether."""
    K = c["beams"]
    return [-1 if g % 5 == 4 else g * K + max(0, i - 1) for g in range(c["groups"]) for i in range(K)]


def _fork_copies(c):
    """Slots of every copy before a write: for each but one of the beams that share a partly filled last page."""
    if not c["n_new"]:
        return []
    lens, parents, P = _fork_lens(c), _parents(c), c["page"]
    own, copies = set(), []
    for p in parents:
        if p < 0 or lens[p] % P == 0:
            continue
        last = _fork_page(c, p, lens[p] // P)
        if last in own:
            copies.append(lens[p] % P)
        own.add(last)
    return copies


def _fork_page(c, row, i):
    """What page i of a beam is, before the pages are numbered: the sample's where it lies in the prompt, else the beam's."""
    return (row // c["beams"], -1, i) if (i + 1) * c["page"] <= c["prompt"] else (row // c["beams"], row, i)


def _fork_pages(c):
    return len({_fork_page(c, r, i) for r, n in enumerate(_fork_lens(c)) for i in range(-(-n // c["page"]))})


def _pool(c):
    """Bytes of one cache (keys or values) of a case."""
    if c["kind"] == "beam":
        return 0
    one = c["page"] * c["Hkv"] * c["dh"] * _size(c["dtype"])
    if c["kind"] == "fork":
        rows = c["groups"] * c["beams"]
        return c["L"] * one * (_fork_pages(c) + rows * (2 + c["n_new"] // c["page"]) + 7)
    return one * sum(-(-n // c["page"]) + 1 for n in _lens(c))


def work(c):
    es = _size(c["dtype"])
    if c["kind"] == "rope":
        N = sum(_news(c))
        byts = N * (2 * c["H"] + 4 * c["Hkv"]) * c["dh"] * es + 4 * N * c["axes"]
        return {"bytes": float(byts), "flops": 3.0 * N * (c["H"] + c["Hkv"]) * c["rot"]}
    if c["kind"] == "attn":
        N, slots, pairs = sum(_news(c)), 0, 0
        w = c["window"] or 1 << 60
        for n, t in zip(_lens(c), _news(c)):
            slots += min(n, t - 1 + w)
            full = max(0, min(t, n - w))  # rows that see a whole window; the others see their position + 1 slots
            pairs += full * min(w, n) + sum(range(n - t + 1, n - full + 1)) if full < t else full * w
        return {"bytes": float(2 * slots * c["Hkv"] * c["dh"] * es + 2 * N * c["H"] * c["dh"] * es), "flops": 4.0 * pairs * c["H"] * c["dh"]}
    if c["kind"] == "fork":
        rows = c["groups"] * c["beams"]
        cols = -(-(c["len"] + c["n_new"]) // c["page"])
        pages = _pool(c) // (c["L"] * c["page"] * c["Hkv"] * c["dh"] * es)
        byts = 8 * rows * cols + 16 * rows + 8 * pages + 4 * c["L"] * sum(_fork_copies(c)) * c["Hkv"] * c["dh"] * es
        return {"bytes": float(byts), "flops": 0.0}
    rows = c["B"] * c["K"]
    return {"bytes": float(rows * c["V"] * es + 8 * c["B"] * c["M"] * c["history"]), "flops": 4.0 * rows * c["V"]}


# -------------------------------------------------------------------------------------------------------------- inputs
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _cache(c, n_pages, gen, layers=None):
    """Pages of a cache, [.., n_pages, page, Hkv, dh], their slots in the order of tokens or of heads."""
    lead = (n_pages,) if layers is None else (layers, n_pages)
    t = torch.empty(lead + ((c["Hkv"], c["page"], c["dh"]) if c["heads_first"] else (c["page"], c["Hkv"], c["dh"])), dtype=_dtype(c["dtype"]), device=DEV)
    t.normal_(generator=gen)
    return t.transpose(-3, -2) if c["heads_first"] else t


def _plan(c, rng):
    """Page tables, lengths and row boundaries of a batch whose pages lie anywhere in the pool."""
    lens, news = _lens(c), _news(c)
    counts = [-(-n // c["page"]) for n in lens]
    pool = sum(counts) + len(counts)
    ids = rng.permutation(pool).astype(np.int32)
    table = np.full((c["B"], max(counts) + 1), -1, np.int32)
    for b, n in enumerate(counts):
        table[b, :n] = ids[sum(counts[:b]):sum(counts[:b]) + n]
    return pool, torch.from_numpy(table).to(DEV), _ints(lens), _ints([sum(news[:b]) for b in range(len(news) + 1)])


def _sections(c):
    """Frequencies of each axis: the later axes an equal share, the first one the rest."""
    half, n = c["rot"] // 2, c["axes"]
    return [half - (n - 1) * (half // n)] + [half // n] * (n - 1)


def _tables(c):
    """Frequency and axis of each pair of channels: the axes' frequencies in blocks or in turn."""
    half, n, sec = c["rot"] // 2, c["axes"], _sections(c)
    freq = 10000.0 ** (-2.0 * np.arange(half) / c["rot"])
    if c["inter"]:
        axis = [i % n if i % n and i < n * sec[i % n] else 0 for i in range(half)]
    else:
        axis = np.repeat(np.arange(n), sec)
    return freq, np.asarray(axis, np.uint8)


def prepare(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {"c": c}
    normal = lambda *shape, scale=1.0: (scale * torch.randn(*shape, generator=gen, device=DEV)).to(_dtype(c["dtype"]))
    if c["kind"] in ("rope", "attn"):
        N = sum(_news(c))
        pool, s["table"], s["lens"], s["cu"] = _plan(c, rng)
        s["k_pages"], s["v_pages"] = (_cache(c, pool, gen) for _ in range(2))
        s["q"] = normal(N, c["H"], c["dh"], scale=1.5)
        if c["kind"] == "attn":
            s["out"] = torch.zeros_like(s["q"])
            return s
        s["k"], s["v"] = (normal(N, c["Hkv"], c["dh"]) for _ in range(2))
        # image tiles one after another: their number, and the patch's row and column; a fourth axis counts the tokens
        r = np.concatenate([np.arange(n) for n in _news(c)])
        axes = np.stack([r // PATCHES, r % PATCHES // SIDE, r % SIDE, r])[:c["axes"]] if c["axes"] > 1 else r[None]
        s["pos"] = torch.from_numpy((axes + c["at"] + rng.integers(0, 3)).astype(np.int32)).to(DEV)
        freq, axis = _tables(c)
        s["freq"], s["axis"] = torch.from_numpy(freq).to(DEV), torch.from_numpy(axis).to(DEV)
        s["q_out"] = torch.zeros_like(s["q"])
    elif c["kind"] == "fork":
        lens, P, rows = _fork_lens(c), c["page"], c["groups"] * c["beams"]
        pool = _pool(c) // (c["L"] * P * c["Hkv"] * c["dh"] * _size(c["dtype"]))
        ids, number = rng.permutation(pool), {}
        table = np.full((rows, -(-(max(lens) + c["n_new"]) // P) + 1), -1, np.int32)
        ref = np.zeros(pool, np.int32)
        for r, n in enumerate(lens):
            for i in range(-(-n // P)):
                page = number.setdefault(_fork_page(c, r, i), ids[len(number)])
                table[r, i] = page
                ref[page] += 1
        s["table"], s["ref"] = torch.from_numpy(table).to(DEV), torch.from_numpy(ref).to(DEV)
        s["lens"], s["parent"], s["n_new"] = _ints(lens), _ints(_parents(c)), _ints([c["n_new"]] * rows)
        s["k"], s["v"] = (_cache(c, pool, gen, c["L"]) for _ in range(2))
        s["table_out"], s["ref_out"], s["lens_out"] = torch.empty_like(s["table"]), torch.empty_like(s["ref"]), torch.empty_like(s["lens"])
    else:
        B, K, V, n = c["B"], c["K"], c["V"], c["history"]
        s["logits"] = normal(B, K, V, scale=2.5)
        s["scores"] = -5.0 * torch.rand(B, K, generator=gen, device=DEV) - 20.0
        s["done"] = _ints(rng.integers(0, 4, (B, K)) == 0) if c["done"] else None
        s["history"] = torch.from_numpy(rng.integers(0, V, (B * K, n + 16)).astype(np.int32)).to(DEV)
        s["n_history"] = _ints([n - (b * 37) % (n // 3 + 1) for b in range(B) for _ in range(K)])
        s["history_out"] = torch.zeros(B * c["M"], n + 16, dtype=torch.int32, device=DEV)
    return s


# --------------------------------------------------------------------------------------------------------- plain forms
def _plain_rope(s):
    c = s["c"]
    half, P = c["rot"] // 2, c["page"]
    angle = s["pos"].double()[s["axis"].long()].t() * s["freq"]                            # [N, half]
    cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))

    def turned(x):
        x = x.float()
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1).to(s["q"].dtype)

    cu, news = s["cu"].long(), s["cu"][1:] - s["cu"][:-1]
    r = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(cu, r, right=True) - 1
    slot = (s["lens"] - news).long()[b] + r - cu[b]
    page = s["table"].long()[b, slot // P]
    s["k_pages"][page, slot % P] = turned(s["k"])
    s["v_pages"][page, slot % P] = s["v"]
    return {"q": turned(s["q"]), "k": s["k_pages"], "v": s["v_pages"]}


def _plain_attn(s):
    c = s["c"]
    H, Hkv, dh, P = c["H"], c["Hkv"], c["dh"], c["page"]
    G, at, out = H // Hkv, 0, torch.zeros_like(s["q"])
    for b, (n, t) in enumerate(zip(_lens(c), _news(c))):
        j = torch.arange(n, device=DEV)
        page = s["table"][b, j // P].long()
        pos = torch.arange(n - t, n, device=DEV)[:, None]
        hidden = j > pos
        if c["window"]:
            hidden = hidden | (j <= pos - c["window"])
        step = max(1, min(Hkv, int(1e9 // (t * G * n))))
        for h in range(0, Hkv, step):
            m = min(step, Hkv - h)
            k, v = (x[page, j % P, h:h + m].float().transpose(0, 1).contiguous() for x in (s["k_pages"], s["v_pages"]))   # [m, n, dh]
            q = s["q"][at:at + t, h * G:(h + m) * G].float().view(t, m, G, dh).permute(1, 0, 2, 3).reshape(m, t * G, dh)
            x = torch.matmul(q, k.transpose(1, 2).contiguous()).view(m, t, G, n).mul_(dh ** -0.5)
            x.masked_fill_(hidden[None, :, None], -math.inf)
            x.sub_(x.amax(-1, keepdim=True)).exp_()
            x.div_(x.sum(-1, keepdim=True))
            o = torch.matmul(x.view(m, t * G, n), v).view(m, t, G, dh)
            out[at:at + t, h * G:(h + m) * G] = o.permute(1, 0, 2, 3).reshape(t, m * G, dh).to(out.dtype)
        at += t
    return {"out": out}


def _plain_fork(s):
    c, table, lens, parent, n_new = s["c"], s["table"].long(), s["lens"].long(), s["parent"].long(), s["n_new"].long()
    P, (rows, M), pool = c["page"], table.shape, s["ref"].shape[0]
    i = torch.arange(M, device=DEV)
    lives = parent >= 0
    n = torch.where(lives, lens[parent.clamp(min=0)], torch.zeros_like(parent))
    grown = torch.where(lives, n + n_new, torch.zeros_like(n))
    pages, pages_grown = (n + P - 1) // P, (grown + P - 1) // P
    new = torch.where(i < pages[:, None], table[parent.clamp(min=0)], -1)
    before = torch.where(i < ((lens + P - 1) // P)[:, None], table, -1)
    ref = s["ref"].long()
    for t, sign in ((before, -1), (new, 1)):
        held = (t >= 0).long().flatten()
        ref = ref.scatter_add(0, t.clamp(min=0).flatten(), sign * held)
    # beams that write into a partly filled page: all but the first take a copy, the first too if others hold the page
    last = torch.gather(new, 1, (n // P).clamp(max=M - 1)[:, None])[:, 0]
    writes = lives & (grown > n) & (n % P > 0) & (last >= 0)
    same = (last[:, None] == last[None]) & writes[:, None] & writes[None]
    first = ~(same & (torch.arange(rows, device=DEV)[None] < torch.arange(rows, device=DEV)[:, None])).any(1)
    copies = writes & ~(first & (ref[last.clamp(min=0)] == same.sum(1)))
    ref = ref.scatter_add(0, last.clamp(min=0), -copies.long())
    free = torch.sort(torch.where(ref <= 0, torch.arange(pool, device=DEV), pool)).values
    need = copies.long() + pages_grown - pages
    start = torch.cumsum(need, 0) - need
    order = torch.where(copies[:, None] & (i == (n // P)[:, None]), start[:, None], -1)
    order = torch.where((i >= pages[:, None]) & (i < pages_grown[:, None]), (start + copies.long() - pages)[:, None] + i, order)
    given = torch.where(order >= 0, free[order.clamp(0, pool - 1)], -1)
    missing = ((order >= 0) & ((order >= pool) | (given == pool))).sum()
    given = torch.where((order >= pool) | (given == pool), -1, given)
    out = torch.where(order >= 0, given, new)
    ref = torch.where(torch.zeros(pool + 1, dtype=torch.bool, device=DEV).scatter_(0, torch.where(given >= 0, given, pool).flatten(), True)[:pool], 1, ref)
    r = torch.nonzero(copies)[:, 0]
    src, dst = last[r], out[r, (n // P)[r]]
    moves = (torch.arange(P, device=DEV)[None] < (n % P)[r][:, None])[None, :, :, None, None]
    for x in (s["k"], s["v"]):
        x[:, dst] = torch.where(moves, x[:, src], x[:, dst])
    return {"table": out.int(), "lens": grown.int(), "ref": ref.int(), "missing": missing.int().view(1), "k": s["k"], "v": s["v"]}


def _plain_beam(s):
    c = s["c"]
    B, K, V, M = c["B"], c["K"], c["V"], c["M"]
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    x = s["scores"].double()[..., None] + (x - (top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))))
    ids = torch.arange(V, device=DEV)
    done = torch.zeros(B, K, dtype=torch.bool, device=DEV) if s["done"] is None else s["done"] > 0
    if c["done"]:
        x = torch.where(done[..., None], torch.where(ids == c["eos"], s["scores"].double()[..., None], -math.inf), x)
    x = x.view(B, K * V)
    place = torch.arange(K * V, device=DEV)
    best, at = [], []
    for _ in range(M):
        best.append(x.amax(-1, keepdim=True))
        at.append(torch.where(x == best[-1], place, K * V).amin(-1, keepdim=True))
        x = x.scatter(1, at[-1], -math.inf)
    at = torch.cat(at, 1)
    beam, token = at // V, at % V
    ended = torch.gather(done, 1, beam)
    parent = (beam + K * torch.arange(B, device=DEV)[:, None]).flatten()
    n = s["n_history"].long()[parent]
    cap = s["history"].shape[1]
    col = torch.arange(cap, device=DEV)
    out = torch.where(col < n[:, None], s["history"][parent], s["history_out"])
    out = torch.where((col == n[:, None]) & ~ended.view(-1, 1), token.view(-1, 1).int(), out)
    grown = torch.where(ended.flatten(), n, (n + 1).clamp(max=cap))
    return {"scores": torch.cat(best, 1).float(), "parent": parent.view(B, M).int(), "token": token.int(),
            "done": (ended | ((token == c["eos"]) if c["eos"] >= 0 else False)).int(), "history": out, "n_history": grown.int()}


# ------------------------------------------------------------------------------------------------------------ one pass
def run(s):
    kind = s["c"]["kind"]
    if not own:
        return {"rope": _plain_rope, "attn": _plain_attn, "fork": _plain_fork, "beam": _plain_beam}[kind](s)
    from paper_2609_34977_amd import _lib
    if kind == "rope":
        q = _lib.rope_append(s["pos"], s["freq"], s["axis"], q=s["q"], q_out=s["q_out"], k=s["k"], v=s["v"], k_pages=s["k_pages"], v_pages=s["v_pages"],
                             table=s["table"], lens=s["lens"], cu_q=s["cu"])
        return {"q": q, "k": s["k_pages"], "v": s["v_pages"]}
    if kind == "attn":
        return {"out": _lib.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["cu"], window=s["c"]["window"], out=s["out"])}
    if kind == "fork":
        table, lens, ref, missing = _lib.pages_fork(s["k"], s["v"], s["table"], s["lens"], s["ref"], s["parent"], n_new=s["n_new"],
                                                    table_out=s["table_out"], lens_out=s["lens_out"], ref_out=s["ref_out"])
        return {"table": table, "lens": lens, "ref": ref, "missing": missing, "k": s["k"], "v": s["v"]}
    return _lib.beam_select(s["logits"], s["scores"], s["c"]["M"], done=s["done"], eos=s["c"]["eos"], history=s["history"], n_history=s["n_history"],
                            history_out=s["history_out"])


# ------------------------------------------------------------------------------------------------------------- 64 bits
def _slots(c, s, b, n):
    """(page, place in it) of the first n slots of sequence b."""
    j = np.arange(n)
    return torch.from_numpy(s["table"][b].cpu().numpy().astype(np.int64)[j // c["page"]]).to(DEV), torch.from_numpy(j % c["page"]).to(DEV)


def _exact_rope(s):
    c, at = s["c"], 0
    half = c["rot"] // 2
    freq, axis = _tables(c)
    pos = s["pos"].cpu().numpy().astype(np.float64)
    q, kp, vp = s["q"].double(), s["k_pages"].double(), s["v_pages"].double()
    k = s["k"].double()
    unit = torch.from_numpy(np.exp(1j * pos[axis.astype(int)].T * freq)).to(DEV)[:, None]  # [N, 1, half]
    for x in (q, k):
        z = torch.complex(x[..., :half], x[..., half:2 * half]) * unit
        x[..., :half], x[..., half:2 * half] = z.real, z.imag
    for b, (n, t) in enumerate(zip(_lens(c), _news(c))):
        page, place = (x[n - t:] for x in _slots(c, s, b, n))
        kp[page, place], vp[page, place] = k[at:at + t], s["v"][at:at + t].double()
        at += t
    return {"q": q, "k": kp, "v": vp}


def _exact_attn(s):
    c, at, out = s["c"], 0, s["q"].double()
    G = c["H"] // c["Hkv"]
    for b, (n, t) in enumerate(zip(_lens(c), _news(c))):
        page, place = _slots(c, s, b, n)
        last = torch.arange(n - t, n, device=DEV)
        sees = torch.ones(t, n, dtype=torch.bool, device=DEV).tril(n - t)
        if c["window"]:
            sees &= torch.arange(n, device=DEV)[None] + c["window"] > last[:, None]
        for h in range(c["H"]):
            K, V = s["k_pages"][page, place, h // G].double(), s["v_pages"][page, place, h // G].double()
            for r in range(0, t, 2048):
                x = (out[at + r:at + min(t, r + 2048), h] / math.sqrt(c["dh"])) @ K.T
                out[at + r:at + min(t, r + 2048), h] = torch.softmax(x.masked_fill(~sees[r:r + 2048], -math.inf), -1) @ V
        at += t
    return {"out": out}


def _exact_fork(s):
    c = s["c"]
    P, lens = c["page"], _fork_lens(c)
    table, ref = s["table"].cpu().numpy(), s["ref"].cpu().numpy().copy()
    pages = [[] if p < 0 else list(table[p, :-(-lens[p] // P)]) for p in _parents(c)]
    for r, n in enumerate(lens):
        np.subtract.at(ref, table[r, :-(-n // P)], 1)
    for row in pages:
        np.add.at(ref, np.array(row, int), 1)
    writers = [r for r, p in enumerate(_parents(c)) if p >= 0 and c["n_new"] and lens[p] % P]
    lasts = [pages[r][-1] for r in writers]
    held = ref.copy()
    copied = [(r, page) for w, (r, page) in enumerate(zip(writers, lasts)) if page in lasts[:w] or held[page] > lasts.count(page)]
    for _, page in copied:
        ref[page] -= 1
    free = iter(np.flatnonzero(ref <= 0))
    k, v = s["k"].double(), s["v"].double()
    for r, p in enumerate(_parents(c)):
        for page in [page for row, page in copied if row == r]:
            n, to = lens[p] % P, int(next(free))
            for x in (k, v):
                x[:, to, :n] = x[:, int(page), :n]
        for _ in range(-(-(lens[p] + c["n_new"]) // P) - len(pages[r]) if p >= 0 else 0):
            next(free)
    return {"table": None, "lens": None, "ref": None, "missing": None, "k": k, "v": v}


def _exact_beam(s):
    c = s["c"]
    x = s["logits"].cpu().double().numpy()
    scores = s["scores"].cpu().double().numpy()
    out = np.zeros((c["B"], c["M"]))
    for b in range(c["B"]):
        rows = []
        for k in range(c["K"]):
            if c["done"] and s["done"][b, k]:
                rows.append(scores[b, k:k + 1])
            else:
                best = np.sort(np.partition(x[b, k], -c["M"])[-c["M"]:])[::-1]
                rows.append(scores[b, k] + best - (best[0] + math.log(np.exp(x[b, k] - best[0]).sum())))
        out[b] = np.sort(np.concatenate(rows))[::-1][:c["M"]]
    return {"scores": torch.from_numpy(out), "parent": None, "token": None, "done": None, "history": None, "n_history": None}


def exact(c, seed):
    if c["kind"] == "beam" and c["B"] * c["K"] * c["V"] > 1e8:
        return None
    if c["kind"] == "fork" and _pool(c) > 3e9:
        return None
    return {"rope": _exact_rope, "attn": _exact_attn, "fork": _exact_fork, "beam": _exact_beam}[c["kind"]](prepare(c, seed))
