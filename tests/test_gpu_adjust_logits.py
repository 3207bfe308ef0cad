"""spider_adjust_logits against the float64 oracle.

Bar: division or product, product and two differences and one sum, each rounded to fp32
once (half a step, 2^-24 relative to its result), plus n - 1 roundings where n entries
share an id: within 8 * 2^-24 of the largest operand, below 1e-6 * max(20, |x|) for the
values here.  The arg max is the first of the operator's own largest values, exactly, and
agrees with the oracle's wherever that one's two largest are further apart than the bar.
"""
import numpy as np
import pytest
import torch

from oracle import drafting as od
from gpu_common import need_gpu

pytestmark = pytest.mark.gpu


def dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def pack_bits(allowed):
    V = allowed.shape[-1]
    pad = np.zeros(allowed.shape[:-1] + ((V + 31) // 32 * 32,), np.uint8)
    pad[..., :V] = allowed
    return np.packbits(pad, axis=-1, bitorder="little").view(np.int32)


def check(out, nxt, ref, best):
    g = out.double().cpu().numpy()
    live = ~np.isnan(ref)
    fin = live & np.isfinite(ref)
    assert np.array_equal(g[live & ~fin], ref[live & ~fin])
    assert (np.abs(g[fin] - ref[fin]) <= 1e-6 * np.maximum(20.0, np.abs(ref[fin]))).all()
    n = nxt.cpu().numpy()
    for i in np.ndindex(best.shape):
        if best[i] == -2:
            continue
        own = out[i].cpu().numpy()
        own = np.where(np.isnan(own), -np.inf, own)
        assert n[i] == (-1 if own.max() == -np.inf else int(np.argmax(own)))
        top = np.sort(ref[i][~np.isnan(ref[i])])[-2:]
        if best[i] >= 0 and (len(top) < 2 or top[1] - top[0] > 1e-4):
            assert n[i] == best[i]


CASES = [
    # B, T, V, history, dtype, n_bias, mask
    (1, 1, 1, 0, "f32", 0, None),
    (1, 1, 33, 5, "f32", 3, "rows"),
    (3, 1, 500, 60, "bf16", 10, "one"),
    (2, 5, 501, 60, "f32", 40, "rows"),
    (2, 7, 4097, 300, "bf16", 0, None),
    (1, 70, 4096, 100, "f32", 5, "rows"),
    (4, 1, 32000, 700, "f32", 8, "rows"),
    (2, 3, 32064, 1500, "bf16", 300, "rows"),
    (1, 1, 151001, 9000, "f32", 20, "one"),
    (2, 2, 32768, 100, "f32", 600, "rows"),
    (1, 2, 20001, 300, "bf16", 5, "rows"),
    (1, 2, 32769, 100, "bf16", 3, "rows"),
    (1, 1, 65540, 3000, "f32", 1500, None),
    (2, 1, 70001, 50, "bf16", 0, None),
    (1, 3, 4096, 20, "bf16", 2500, "rows"),
    (1, 2, 40004, 20, "f32", 7, "rows"),
    (1, 256, 130, 40, "f32", 2, None),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_adjust_matches_the_oracle(case):
    lib = need_gpu()
    B, T, V, n, dtype, nb, mk = case
    rng = np.random.default_rng(V + T)
    x = torch.from_numpy(rng.normal(0, 3, (B, T, V)).astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    hist = np.minimum(rng.zipf(1.4, (B, n)) - 1, V + 3).astype(np.int32)  # some ids past the vocabulary
    if n:
        hist[0, 0] = -5
    n_hist = np.array([n + 9 if b == 1 else max(0, n - 3 * b) for b in range(B)], np.int32)  # one past the row
    n_prompt = np.array([n // 2 + b for b in range(B)], np.int32)
    nodes = np.array([max(1, T - b) for b in range(B)], np.int32)
    parents = np.stack([np.concatenate([[-1], rng.integers(-1, np.arange(1, T))]) if T > 1 else np.array([-1]) for _ in range(B)])
    sees = od.tree_mask(parents)[0]
    drafted = np.minimum(rng.zipf(1.4, (B, T)) - 1, V).astype(np.int32)
    rep, freq, pres = (rng.uniform(lo, hi, B).astype(np.float32) for lo, hi in ((0.8, 1.5), (-0.2, 0.7), (-0.3, 0.9)))
    ids = rng.integers(-1, V + 2, (B, nb)).astype(np.int32) if nb else None
    if nb > 4:
        ids[:, 3] = ids[:, 1] = ids[:, 4]  # the same token three times
    bias = rng.normal(0, 5, (B, nb)).astype(np.float32) if nb else None
    allowed = None
    if mk == "rows":
        allowed = rng.random((B, T, V)) < 0.5
        allowed[0, 0] = False
        allowed[-1, -1] = False
        allowed[-1, -1, V - 1] = True
    elif mk == "one":
        allowed = rng.random(V) < 0.3
        allowed[V // 2] = True
    out = torch.full((B, T, V), 7.0).cuda()
    nxt = torch.full((B, T), 77, dtype=torch.int32).cuda()
    kw = dict(n_prompt=dev(n_prompt), n_nodes=dev(nodes), node_tokens=dev(drafted), tree_mask=dev(od.pack_mask(sees)),
              repetition=dev(rep), frequency=dev(freq), presence=dev(pres), bias_ids=dev(ids), bias=dev(bias),
              mask=None if allowed is None else dev(pack_bits(allowed)))
    lib.adjust_logits(x.cuda(), dev(hist), dev(n_hist), out=out, next_ids=nxt, **kw)
    ref, best = od.adjust_logits(x.float().numpy(), hist, n_hist, n_prompt, drafted, sees, rep, freq, pres, ids, bias, allowed, nodes)
    check(out, nxt, ref, best)
    dead = best == -2
    assert (out.cpu().numpy()[dead] == 7.0).all() and (nxt.cpu().numpy()[dead] == 77).all()
    again, n2 = lib.adjust_logits(x.cuda(), dev(hist), dev(n_hist), out=torch.full((B, T, V), 7.0).cuda(),
                                  next_ids=torch.full((B, T), 77, dtype=torch.int32).cuda(), **kw)
    assert torch.equal(again, out) and torch.equal(n2, nxt)


def test_a_chain_without_tree_mask_counts_all_earlier_nodes():
    lib = need_gpu()
    rng = np.random.default_rng(1)
    x = rng.normal(0, 2, (2, 9, 200)).astype(np.float32)
    drafted = rng.integers(0, 20, (2, 9)).astype(np.int32)
    freq = np.array([0.5, 0.25], np.float32)
    out, nxt = lib.adjust_logits(dev(x), node_tokens=dev(drafted), frequency=dev(freq))
    check(out, nxt, *od.adjust_logits(x, node_tokens=drafted, frequency=freq))


def test_no_rule_is_the_arg_max_of_the_logits():
    lib = need_gpu()
    x = np.random.default_rng(2).normal(0, 1, (3, 1000)).astype(np.float32)
    x[1] = -np.inf
    x[2, [7, 700]] = 50.0   # a tie: the lower id
    x[0, 10] = np.nan
    out, nxt = lib.adjust_logits(dev(x))
    assert np.array_equal(out.cpu().numpy(), x, equal_nan=True)
    z = np.where(np.isnan(x), -np.inf, x)
    assert nxt.tolist() == [int(np.argmax(z[0])), -1, 7]


@pytest.mark.parametrize("V", [64, 9001])
def test_extreme_values(V):
    """Infinities, NaN and the type's lowest value as logits and as biases."""
    lib = need_gpu()
    low = np.finfo(np.float32).min
    x = np.random.default_rng(3).normal(0, 1, (1, V)).astype(np.float32)
    x[0, :6] = [np.inf, -np.inf, np.nan, low, -low, 0.0]
    hist = np.arange(8, dtype=np.int32)[None]
    ids = np.array([[0, 9, 10, 11, 12, 3]], np.int32)
    bias = np.array([[1.0, -np.inf, low, np.nan, np.inf, low]], np.float32)
    rep = np.array([1.25], np.float32)
    allowed = np.ones(V, bool)
    allowed[[0, 12]] = False
    with np.errstate(all="ignore"):
        ref = x.copy()
        ref[0, :8] = np.where(x[0, :8] > 0, x[0, :8] / rep, x[0, :8] * rep)
        for i, b in zip(ids[0], bias[0]):
            ref[0, i] = ref[0, i] + b
        ref[0, ~allowed] = -np.inf
    out, nxt = lib.adjust_logits(dev(x), dev(hist), dev(np.array([8], np.int32)), repetition=dev(rep), bias_ids=dev(ids),
                                 bias=dev(bias), mask=dev(pack_bits(allowed)))
    assert np.array_equal(out.cpu().numpy(), ref, equal_nan=True)
    assert nxt.item() == 4


def test_in_place_and_strided_rows():
    lib = need_gpu()
    rng = np.random.default_rng(4)
    wide = dev(rng.normal(0, 2, (4, 1003)).astype(np.float32))
    rows = wide[:, 1:902]  # odd distance and start
    pres = dev(np.full(4, 0.5, np.float32))
    hist = dev(rng.integers(0, 901, (4, 50)).astype(np.int32))
    n = dev(np.full(4, 50, np.int32))
    want, ids = lib.adjust_logits(rows.contiguous(), hist, n, presence=pres)
    before = wide.clone()
    out, got = lib.adjust_logits(rows, hist, n, presence=pres, out=rows)
    assert torch.equal(rows, want) and torch.equal(ids, got)
    before[:, 1:902] = want
    assert torch.equal(wide, before)


def test_on_a_stream_and_captured():
    lib = need_gpu()
    rng = np.random.default_rng(5)
    x = dev(rng.normal(0, 2, (2, 3, 5000)).astype(np.float32))
    hist = dev(rng.integers(0, 5000, (2, 400)).astype(np.int32))
    n = dev(np.array([400, 300], np.int32))
    rep = dev(np.array([1.2, 1.1], np.float32))
    drafted = dev(rng.integers(0, 5000, (2, 3)).astype(np.int32))
    call = lambda **k: lib.adjust_logits(x, hist, n, repetition=rep, node_tokens=drafted, **k)  # noqa: E731
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out, ids = torch.empty_like(x), torch.empty(2, 3, dtype=torch.int32).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, next_ids=ids)
    for i in range(3):
        x.copy_(torch.roll(x, 13, 2))
        n.sub_(50)
        graph.replay()
        torch.cuda.synchronize()
        a, b = call()
        assert torch.equal(out, a) and torch.equal(ids, b)


def test_refusals_of_the_binding():
    lib = need_gpu()
    x = torch.zeros(2, 3, 100).cuda()
    hist = torch.zeros(2, 5, dtype=torch.int32).cuda()
    n = torch.zeros(2, dtype=torch.int32).cuda()
    bad = [
        lambda: lib.adjust_logits(x.half()),
        lambda: lib.adjust_logits(x[..., ::2]),
        lambda: lib.adjust_logits(x[:, :2]),
        lambda: lib.adjust_logits(x, hist),
        lambda: lib.adjust_logits(x, hist.long(), n),
        lambda: lib.adjust_logits(x, hist, n.cpu()),
        lambda: lib.adjust_logits(x, repetition=torch.ones(2, dtype=torch.float64).cuda()),
        lambda: lib.adjust_logits(x, bias=torch.ones(2, 4).cuda()),
        lambda: lib.adjust_logits(x, mask=torch.ones(2, 3, 3, dtype=torch.int32).cuda()),
        lambda: lib.adjust_logits(x, tree_mask=torch.ones(2, 3, 2, dtype=torch.int64).cuda()),
        lambda: lib.adjust_logits(x.bfloat16(), out=torch.zeros(2, 3, 99).cuda()),
        lambda: lib.adjust_logits(torch.zeros(2, 40000).cuda(), workspace=torch.empty(8, dtype=torch.uint8).cuda()),
    ]
    for f in bad:
        with pytest.raises((ValueError, TypeError, lib.SpiderError)):
            f()
