"""spider_tree_attention against the float64 oracle.

Bars, derived from the roundings.  fp32: a score is a sum of dh products, off by at
most about dh * 2^-24 of sum |q k| scale (here up to ~10), so a weight is off by
~ dh * 10 * 2^-24 relative at worst and typically by its square root of that; the bar is
2e-5 of the largest output.  bf16: the output is rounded once (half a step, 2^-8 of its own
size), the weights enter with 16 significant bits (2^-16) and the scores are fp32 as above:
2^-8 |out| + 1e-4 of the largest value.  With more than 32 rows per kv head (16 past a dh of
128) the weights are rounded to bf16 once, p (1 + d) with |d| <= 2^-8, so out is off by
|sum p d v| <= 2^-8 sum p |v| more (1 % on top for that term's own rounding).
Weights out are fp32 sums of at most T * G terms: 2e-5 of the largest, plus 1e-6.
"""
import numpy as np
import pytest
import torch

from oracle import drafting as od
from gpu_common import need_gpu

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def trees(B, T, rng):
    p = np.zeros((B, T), np.int32)
    for b in range(B):
        for t in range(T):
            p[b, t] = rng.integers(-1, t) if t and rng.random() < 0.6 else t - 1
    return p


def make(B, T, H, Hkv, dh, cap, dtype, seed, heads_first=False, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    q = (spread * torch.randn(B, T, H, dh, generator=g)).to(DT[dtype]).cuda()
    shape = (B, Hkv, cap, dh) if heads_first else (B, cap, Hkv, dh)
    k, v = (torch.randn(shape, generator=g).to(DT[dtype]).cuda() for _ in range(2))
    if heads_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return q, k, v


def check(got, ref, dtype, mean_abs=None):
    """mean_abs: sum p |v| of every output where the weights are rounded to bf16."""
    g, o = got.double().cpu().numpy(), ref
    live = ~np.isnan(o)
    big = max(np.abs(o[live]).max(), 1e-30) if live.any() else 1.0
    bar = 2e-5 * big if dtype == "f32" else 2.0 ** -8 * np.abs(o[live]) + 1e-4 * big
    if mean_abs is not None:
        bar = bar + 1.01 * 2.0 ** -8 * mean_abs[live]
    assert np.isfinite(g[live]).all()
    err = np.abs(g[live] - o[live])
    assert (err <= bar).all(), (err.max(), big)


def np64(t):
    return t.double().cpu().numpy()


CASES = [
    # B, T, H, Hkv, dh, lens, dtype, heads_first, weights
    (1, 1, 32, 32, 128, [200], "bf16", False, True),
    (2, 1, 4, 4, 128, [0, 1], "bf16", False, True),
    (3, 2, 8, 2, 128, [0, 31, 32], "bf16", True, True),
    (2, 5, 6, 2, 64, [33, 64], "bf16", False, True),
    (2, 16, 4, 4, 128, [705, 127], "bf16", False, True),
    (1, 17, 8, 1, 128, [1000], "bf16", True, True),
    (2, 64, 4, 2, 128, [257, 3], "bf16", False, True),
    (1, 65, 4, 2, 80, [130], "bf16", False, True),
    (1, 130, 2, 2, 256, [70], "bf16", True, True),
    (1, 256, 2, 1, 64, [5], "bf16", False, True),
    (2, 3, 2, 2, 8, [9, 40], "bf16", False, True),
    (1, 7, 16, 2, 96, [5000], "bf16", False, False),
    (1, 1, 8, 1, 256, [3001], "bf16", False, True),
    (1, 33, 12, 4, 40, [513], "bf16", True, False),
    (1, 60, 2, 2, 64, [700], "bf16", False, True),
    (1, 20, 2, 2, 64, [300], "bf16", False, True),
    (1, 5, 4, 2, 96, [300], "bf16", False, True),
    (1, 8, 2, 2, 256, [130], "f32", False, True),
    (1, 100, 2, 2, 64, [333], "bf16", True, False),
    (2, 20, 2, 2, 128, [450, 31], "bf16", False, True),
    (1, 61, 2, 2, 128, [1999], "bf16", True, True),
    (1, 120, 2, 2, 128, [1030], "bf16", False, True),
    (1, 61, 8, 2, 128, [4100], "bf16", True, False),
    (1, 20, 2, 2, 48, [100], "bf16", False, True),
    (1, 50, 2, 2, 56, [90], "bf16", False, True),
    (1, 150, 2, 2, 40, [64], "bf16", False, True),
    (1, 24, 2, 2, 104, [200], "bf16", False, True),
    (1, 50, 2, 2, 120, [31], "bf16", False, True),
    (1, 100, 2, 2, 72, [77], "bf16", False, True),
    (1, 200, 4, 2, 112, [95], "bf16", False, True),
    (1, 10, 2, 2, 256, [800], "bf16", False, True),
    (1, 30, 2, 2, 256, [400], "bf16", False, True),
    (1, 9, 2, 2, 200, [100], "bf16", False, True),
    (1, 20, 2, 2, 136, [100], "bf16", False, True),
    (1, 60, 2, 2, 248, [64], "bf16", False, True),
    (1, 30, 2, 2, 128, [200], "f32", False, True),
    (1, 10, 2, 2, 100, [200], "f32", False, True),
    (1, 40, 2, 2, 100, [130], "f32", False, True),
    (1, 40, 2, 2, 256, [130], "f32", False, True),
    (1, 9, 2, 2, 132, [130], "f32", False, True),
    (1, 40, 2, 2, 252, [130], "f32", False, True),
    (1, 30, 2, 2, 64, [500], "f32", True, True),
    (2, 13, 8, 8, 64, [1500, 1001], "f32", False, True),
    (2, 1, 4, 2, 32, [0, 99], "f32", False, True),
    (1, 70, 6, 2, 48, [61], "f32", True, True),
    (1, 9, 4, 1, 256, [300], "f32", False, True),
    (1, 2, 3, 3, 4, [17], "f32", False, True),
    (1, 200, 2, 1, 128, [2], "f32", False, True),
    (1, 1, 16, 2, 128, [9000], "f32", False, True),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_tree_attention_matches_the_oracle(case):
    lib = need_gpu()
    B, T, H, Hkv, dh, lens, dtype, heads_first, weighted = case
    rng = np.random.default_rng(T * 1000 + dh)
    cap = max(lens) + T + 5
    q, k, v = make(B, T, H, Hkv, dh, cap, dtype, T + dh, heads_first, 1.5)
    mask, _ = lib.tree_mask(trees(B, T, rng))
    sees = od.tree_mask(trees(B, T, np.random.default_rng(T * 1000 + dh)))[0]
    nodes = [max(0, T - 2 * b) for b in range(B)]
    w_in = torch.rand(B, Hkv, cap).cuda() if weighted else None
    w_out = torch.full((B, Hkv, cap), -7.0).cuda() if weighted else None
    out = torch.full_like(q, 9.0)
    args = dict(n_nodes=torch.tensor(nodes, dtype=torch.int32).cuda(), tree_mask=torch.from_numpy(mask).cuda(), out=out,
                weights_in=w_in, weights_out=w_out)
    ln = torch.tensor(lens, dtype=torch.int32).cuda()
    lib.tree_attention(q, k, v, ln, **args)
    ref, wref = od.tree_attention(np64(q), np64(k), np64(v), lens, sees, nodes, weights_in=np64(w_in) if weighted else None)
    many = dtype == "bf16" and T * H // Hkv > (16 if dh > 128 else 32)
    check(out, ref, dtype, od.tree_attention(np64(q), np64(k), np.abs(np64(v)), lens, sees, nodes)[0] if many else None)
    assert (out.float().cpu().numpy()[np.isnan(ref)] == 9.0).all()  # rows of nodes that are not alive
    if weighted:
        w = np64(w_out)
        live = ~np.isnan(wref)
        assert (w[~live] == -7.0).all()
        if live.any():
            assert np.abs(w[live] - wref[live]).max() <= 2e-5 * wref[live].max() + 1e-6
    first = out.clone(), (w_out.clone() if weighted else None)
    lib.tree_attention(q, k, v, ln, **args)
    assert torch.equal(out, first[0]) and (not weighted or torch.equal(w_out, first[1]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_chain_without_mask_is_the_causal_mask(dtype):
    lib = need_gpu()
    q, k, v = make(2, 40, 4, 2, 128, 200, dtype, 3)
    ln = torch.tensor([150, 0], dtype=torch.int32).cuda()
    sees = np.broadcast_to(np.tril(np.ones((40, 40), bool)), (2, 40, 40))
    out = lib.tree_attention(q, k, v, ln)
    masked = lib.tree_attention(q, k, v, ln, tree_mask=torch.from_numpy(od.pack_mask(sees)).cuda())
    assert torch.equal(out, masked)
    mean_abs = od.tree_attention(np64(q), np64(k), np.abs(np64(v)), [150, 0])[0] if dtype == "bf16" else None
    check(out, od.tree_attention(np64(q), np64(k), np64(v), [150, 0])[0], dtype, mean_abs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing_are_zero(dtype):
    lib = need_gpu()
    q, k, v = make(2, 6, 4, 2, 64, 40, dtype, 4)
    sees = np.zeros((2, 6, 6), bool)
    sees[:, 3, 1] = True
    sees[:, 5, 5] = True
    w_out = torch.full((2, 2, 40), -1.0).cuda()
    ln = torch.tensor([0, 0], dtype=torch.int32).cuda()
    out = lib.tree_attention(q, k, v, ln, tree_mask=torch.from_numpy(od.pack_mask(sees)).cuda(), weights_out=w_out)
    ref, wref = od.tree_attention(np64(q), np64(k), np64(v), [0, 0], sees)
    assert (out[:, [0, 1, 2, 4]] == 0).all()
    check(out, ref, dtype)
    assert np.abs(np64(w_out)[:, :, :6] - wref[:, :, :6]).max() <= 1e-6
    assert (w_out[:, :, 6:] == -1).all()


@pytest.mark.parametrize("T", [6, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_hidden_slots_hold_does_not_count(dtype, bad, T):
    """Slots past the live nodes, nodes nobody sees and nodes that only some rows see."""
    lib = need_gpu()
    q, k, v = make(1, T, 4, 2, 128, 128, dtype, 5)
    sees = np.tril(np.ones((1, T, T), bool))
    sees[0, :, 2] = False           # seen by nobody
    sees[0, 4:, 1] = False          # seen by rows 1..3 only
    n = 50
    ln = torch.tensor([n], dtype=torch.int32).cuda()
    mask = torch.from_numpy(od.pack_mask(sees)).cuda()
    nodes = torch.tensor([T - 1], dtype=torch.int32).cuda()
    w, w2 = torch.zeros(1, 2, 128).cuda(), torch.zeros(1, 2, 128).cuda()
    clean = lib.tree_attention(q, k, v, ln, tree_mask=mask, n_nodes=nodes, out=torch.zeros_like(q), weights_out=w)
    k2, v2 = k.clone(), v.clone()
    k2[:, n + 2], v2[:, n + 2] = bad, bad
    k2[:, n + T - 1:], v2[:, n + T - 1:] = bad, bad
    v2[:, n + 1, 0, 3::7] = bad
    k2[:, n + 1, 1] = bad
    got = lib.tree_attention(q, k2, v2, ln, tree_mask=mask, n_nodes=nodes, out=torch.zeros_like(q), weights_out=w2)
    assert torch.equal(got[:, [0] + list(range(4, T))], clean[:, [0] + list(range(4, T))])
    # rows 1..3 see it: the first kv head's channels 3, 10, .. of v, the second's whole row through k
    seen = got[0, 1:4, :2, 3::7].float()
    assert (torch.isnan(seen) if bad != bad else seen == bad).all()
    rest = [c for c in range(128) if c % 7 != 3]
    assert torch.equal(got[0, 1:4, :2][:, :, rest], clean[0, 1:4, :2][:, :, rest])
    assert torch.equal(w[:, 0, :n], w2[:, 0, :n])


def test_strides_of_a_packed_projection_and_a_layer_of_a_cache():
    lib = need_gpu()
    B, T, H, Hkv, dh, L, cap = 2, 3, 4, 2, 64, 3, 70
    g = torch.Generator().manual_seed(6)
    packed = torch.randn(B, T + 2, (H + 2 * Hkv) * dh, generator=g).bfloat16().cuda()
    q = packed[:, 1:T + 1, :H * dh].unflatten(2, (H, dh))
    cache = torch.randn(2, L, B, cap + 3, Hkv + 1, dh + 8, generator=g).bfloat16().cuda()
    k, v = (cache[i, 1, :, 2:cap + 2, 1:, :dh] for i in range(2))
    ln = torch.tensor([60, 11], dtype=torch.int32).cuda()
    out = lib.tree_attention(q, k, v, ln)
    assert torch.equal(out, lib.tree_attention(q.contiguous(), k.contiguous(), v.contiguous(), ln))
    check(out, od.tree_attention(np64(q), np64(k), np64(v), [60, 11])[0], "bf16")


def test_lengths_outside_the_cache_are_taken_into_it():
    lib = need_gpu()
    q, k, v = make(4, 3, 2, 2, 64, 50, "bf16", 7)
    lens = [-5, 49, 50, 1000]
    out = torch.full_like(q, 2.0)
    lib.tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32).cuda(), out=out)
    ref, _ = od.tree_attention(np64(q), np64(k), np64(v), lens)
    check(out, ref, "bf16")
    assert (out.float().cpu().numpy()[np.isnan(ref)] == 2.0).all()


def test_node_counts_outside_the_tree_are_taken_into_it():
    lib = need_gpu()
    q, k, v = make(3, 4, 2, 2, 64, 50, "bf16", 8)
    out = torch.full_like(q, 2.0)
    lib.tree_attention(q, k, v, torch.tensor([9, 9, 9], dtype=torch.int32).cuda(), out=out,
                       n_nodes=torch.tensor([-1, 99, 0], dtype=torch.int32).cuda())
    ref, _ = od.tree_attention(np64(q), np64(k), np64(v), [9, 9, 9], n_nodes=[-1, 99, 0])
    check(out, ref, "bf16")
    assert (out[0] == 2).all() and (out[2] == 2).all()


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 40), ("bf16", 128), ("bf16", 96), ("f32", 64), ("f32", 36),
                                      ("f32", 128), ("f32", 100)])
def test_weights_of_many_rows_over_many_heads(dtype, dh):
    """Enough blocks for the weights pass that takes two tiles of keys at a time."""
    lib = need_gpu()
    B, T, Hkv, cap = 8, 9, 16, 1100 if dtype == "bf16" else 600
    lens = [cap - 10 - 97 * b % 500 for b in range(B)]
    q, k, v = make(B, T, 2 * Hkv, Hkv, dh, cap, dtype, 17, spread=1.5)
    w_in, w_out = torch.rand(B, Hkv, cap).cuda(), torch.full((B, Hkv, cap), -7.0).cuda()
    lib.tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32).cuda(), weights_in=w_in, weights_out=w_out)
    _, ref = od.tree_attention(np64(q), np64(k), np64(v), lens, weights_in=np64(w_in))
    live = ~np.isnan(ref)
    assert (np64(w_out)[~live] == -7.0).all()
    assert np.abs(np64(w_out)[live] - ref[live]).max() <= 2e-5 * ref[live].max() + 1e-6


@pytest.mark.parametrize("T", [2, 40])
def test_samples_without_nodes_pass_their_weights_on(T):
    """No live node, over one tile and over many splits: the context's weights go through unchanged."""
    lib = need_gpu()
    q, k, v = make(3, T, 4, 2, 64, 3100, "bf16", 13)
    lens, nodes = [3000, 20, 3000], [0, 0, 1]
    w_in, w_out = torch.rand(3, 2, 3100).cuda(), torch.full((3, 2, 3100), -2.0).cuda()
    out = torch.full_like(q, 2.0)
    lib.tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32).cuda(), out=out, weights_in=w_in, weights_out=w_out,
                       n_nodes=torch.tensor(nodes, dtype=torch.int32).cuda())
    for b in (0, 1):
        assert torch.equal(w_out[b, :, :lens[b]], w_in[b, :, :lens[b]]) and (w_out[b, :, lens[b]:] == -2).all()
    assert (out[:2] == 2).all()
    ref, wref = od.tree_attention(np64(q), np64(k), np64(v), lens, n_nodes=nodes, weights_in=np64(w_in))
    mean_abs = od.tree_attention(np64(q), np64(k), np.abs(np64(v)), lens, n_nodes=nodes)[0]
    check(out, ref, "bf16", mean_abs)
    assert np.abs(np64(w_out)[2, :, :3001] - wref[2, :, :3001]).max() <= 2e-5


@pytest.mark.parametrize("dtype,T", [("bf16", 3), ("bf16", 50), ("f32", 3), ("f32", 30)])
@pytest.mark.parametrize("scale", [-0.2, 0.0])
def test_scales_of_any_sign(scale, dtype, T):
    lib = need_gpu()
    q, k, v = make(1, T, 4, 2, 64, 900, dtype, 14)
    w = torch.zeros(1, 2, 900).cuda()
    out = lib.tree_attention(q, k, v, torch.tensor([800], dtype=torch.int32).cuda(), scale=scale, weights_out=w)
    ref, wref = od.tree_attention(np64(q), np64(k), np64(v), [800], scale=scale)
    mean_abs = od.tree_attention(np64(q), np64(k), np.abs(np64(v)), [800], scale=scale)[0] if dtype == "bf16" else None
    check(out, ref, dtype, mean_abs)
    live = ~np.isnan(wref)
    assert np.abs(np64(w)[live] - wref[live]).max() <= 2e-5 * wref[live].max() + 1e-6


@pytest.mark.parametrize("T", [3, 50])
def test_two_calls_at_once_on_two_streams(T):
    lib = need_gpu()
    args = [make(2, T, 8, 2, 128, 2000, "bf16", s) for s in (15, 16)]
    ln = torch.tensor([1900, 333], dtype=torch.int32).cuda()
    want = [lib.tree_attention(*a, ln) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, a in zip(streams, args):
            with torch.cuda.stream(s):
                got.append(lib.tree_attention(*a, ln))
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_large_scores_keep_the_softmax_exact():
    """Scores in the hundreds, the largest late in the cache."""
    lib = need_gpu()
    q, k, v = make(1, 4, 2, 1, 128, 3000, "f32", 9, spread=1.0)
    k[0, 2500, 0] = q[0, 2, 1] * 3
    k[0, 100] *= 20
    ln = torch.tensor([2900], dtype=torch.int32).cuda()
    out = lib.tree_attention(q, k, v, ln, scale=0.5)
    ref, _ = od.tree_attention(np64(q), np64(k), np64(v), [2900], scale=0.5)
    # scores up to ~500 in fp32: off by up to 128 * 2^-24 * 1000 absolute, so weights by 8e-3 at worst
    g = np64(out)
    assert np.isfinite(g).all() and np.abs(g - ref).max() <= 8e-3 * np.abs(ref).max()


def test_a_cache_past_four_gigabytes():
    """Two samples a stride of more than 2^32 bytes apart, and slots far into a sample."""
    lib = need_gpu()
    cap, Hkv, dh = 300000, 32, 128
    k = torch.zeros(2, cap, Hkv, dh, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    n = 299000
    lens = [n, n - 7]
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in (k, v):
        x[:, :].normal_(generator=g)
    q = torch.randn(2, 2, 32, dh, generator=g, device="cuda").bfloat16()
    ln = torch.tensor(lens, dtype=torch.int32).cuda()
    w = torch.zeros(2, Hkv, cap, device="cuda")
    out = lib.tree_attention(q, k, v, ln, weights_out=w)
    for h in (0, 31):
        ref, wref = od.tree_attention(np64(q[1:, :, h:h + 1]), np64(k[1:, :, h:h + 1]), np64(v[1:, :, h:h + 1]), lens[1:])
        check(out[1:, :, h:h + 1], ref, "bf16")
        live = ~np.isnan(wref[0, 0])
        assert np.abs(np64(w[1, h])[live] - wref[0, 0][live]).max() <= 1e-6


def test_on_a_stream_and_captured():
    lib = need_gpu()
    q, k, v = make(2, 9, 8, 2, 128, 600, "bf16", 11)
    ln = torch.tensor([500, 77], dtype=torch.int32).cuda()
    w = torch.zeros(2, 2, 600).cuda()
    want, ww = lib.tree_attention(q, k, v, ln, weights_out=w).clone(), w.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lib.tree_attention(q, k, v, ln, weights_out=w)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(w, ww)
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.tree_attention(q, k, v, ln, out=out, weights_out=w)
    for i in range(3):
        ln.copy_(torch.tensor([500 - 100 * i, 77 + i], dtype=torch.int32))
        q.add_(0.25)
        out.zero_(), w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        w2 = torch.zeros_like(w)
        eager = lib.tree_attention(q, k, v, ln, weights_out=w2)
        assert torch.equal(out, eager) and torch.equal(w, w2)


def test_refusals_of_the_binding():
    lib = need_gpu()
    q, k, v = make(2, 3, 4, 2, 64, 50, "bf16", 12)
    ln = torch.tensor([9, 9], dtype=torch.int32).cuda()
    bad = [
        lambda: lib.tree_attention(q, k, v.float(), ln),
        lambda: lib.tree_attention(q, k[:1], v[:1], ln),
        lambda: lib.tree_attention(q, k, v, ln.long()),
        lambda: lib.tree_attention(q, k, v, ln.cpu()),
        lambda: lib.tree_attention(q, k, v, ln[:1]),
        lambda: lib.tree_attention(q[..., ::2], k[..., ::2], v[..., ::2], ln),
        lambda: lib.tree_attention(q, k, v, ln, out=torch.empty(2, 3, 4, 64).cuda()),
        lambda: lib.tree_attention(q, k, v, ln, weights_in=torch.zeros(2, 2, 50).cuda()),
        lambda: lib.tree_attention(q, k, v, ln, weights_out=torch.zeros(2, 2, 49).cuda()),
        lambda: lib.tree_attention(q, k, v, ln, tree_mask=torch.zeros(2, 3, 2, dtype=torch.int64).cuda()),
        lambda: lib.tree_attention(q[:, :, :3], k, v, ln),
        lambda: lib.tree_attention(q[..., :12].contiguous(), k[..., :12], v[..., :12], ln),
        lambda: lib.tree_attention(q.half(), k.half(), v.half(), ln),
        lambda: lib.tree_attention(q, k, v, ln, workspace=torch.empty(16, dtype=torch.uint8).cuda(),
                                   weights_out=torch.zeros(2, 2, 50).cuda()),
    ]
    for f in bad:
        with pytest.raises((ValueError, TypeError, lib.SpiderError)):
            f()
