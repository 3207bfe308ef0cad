"""spider_tree_attention at its edges, against the float64 oracle: splits of the keys that a
ceiling leaves without a tile, hidden infinities and NaN in many tiles, infinite values that count, many rows.

Bars as in test_gpu_tree_attention.py.
"""
import numpy as np
import pytest
import torch

from oracle import drafting as od
from gpu_common import need_gpu
from test_gpu_tree_attention import check, make, np64, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H,dh", [(61, 2, 128), (50, 4, 128), (70, 4, 128), (40, 4, 64), (20, 2, 256), (40, 2, 256)])
@pytest.mark.parametrize("n", [2561, 2592])
def test_splits_that_the_tiles_do_not_fill(n, T, H, dh):
    """81 tiles of keys in at most ten splits of nine: nine of them, in every block width of many rows."""
    lib = need_gpu()
    q, k, v = make(1, T, H, 2, dh, n + 30, "bf16", n + T, spread=1.5)
    rng = np.random.default_rng(T)
    parents = trees(1, T, rng)
    mask, sees = lib.tree_mask(parents)[0], od.tree_mask(parents)[0]
    ln = torch.tensor([n - T], dtype=torch.int32).cuda()
    w = torch.zeros(1, 2, n + 30).cuda()
    out = lib.tree_attention(q, k, v, ln, tree_mask=torch.from_numpy(mask).cuda(), weights_out=w)
    ref, wref = od.tree_attention(np64(q), np64(k), np64(v), [n - T], sees)
    check(out, ref, "bf16", od.tree_attention(np64(q), np64(k), np.abs(np64(v)), [n - T], sees)[0])
    assert np.abs(np64(w)[:, :, :n] - wref[:, :, :n]).max() <= 2e-5 * wref[:, :, :n].max() + 1e-6


def same(a, b):
    """Equal bit for bit, NaN where NaN."""
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("dtype,T,H,dh", [
    ("bf16", 30, 2, 128), ("bf16", 110, 2, 128), ("bf16", 250, 2, 128), ("bf16", 61, 2, 128), ("bf16", 110, 2, 64),
    ("bf16", 200, 4, 40), ("bf16", 110, 2, 256), ("bf16", 250, 1, 200), ("f32", 200, 2, 64), ("f32", 256, 1, 100),
    ("f32", 220, 2, 256)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_hidden_slots_in_many_tiles_do_not_count(bad, dtype, T, H, dh):
    """Bad nodes that nobody sees in every second tile of keys of the tree, one that the last row alone sees, and one
    bad value of the context in the tile that it shares with the tree: all else keeps its bits."""
    lib = need_gpu()
    Hkv, n = min(H, 2), 50
    q, k, v = make(1, T, H, Hkv, dh, n + T + 9, dtype, T + dh)
    hidden = list(range(3, T - 2, 16))
    sees = np.tril(np.ones((1, T, T), bool))
    sees[0, :, hidden] = False
    once = T - 3
    sees[0, :, once] = False
    sees[0, T - 1, once] = True
    mask = torch.from_numpy(od.pack_mask(sees)).cuda()
    ln = torch.tensor([n], dtype=torch.int32).cuda()
    w, w2 = (torch.zeros(1, Hkv, n + T + 9).cuda() for _ in range(2))
    clean = lib.tree_attention(q, k, v, ln, tree_mask=mask, weights_out=w).float()
    k2, v2 = k.clone(), v.clone()
    at = torch.tensor([n + u for u in hidden]).cuda()
    k2[:, at], v2[:, at] = bad, bad
    v2[:, n + once, 0, 1] = bad
    v2[:, 40, 0, 2] = bad
    got = lib.tree_attention(q, k2, v2, ln, tree_mask=mask, weights_out=w2).float()
    G = H // Hkv
    clean[:, T - 1, :G, 1] = bad
    clean[:, :, :G, 2] = bad
    assert same(got, clean)
    assert torch.equal(w, w2)


@pytest.mark.parametrize("dtype,T,H,dh", [
    ("bf16", 1, 2, 128), ("bf16", 5, 2, 128), ("bf16", 5, 2, 64), ("bf16", 20, 2, 96), ("bf16", 9, 2, 256),
    ("bf16", 40, 2, 128), ("bf16", 70, 4, 128), ("bf16", 150, 2, 56), ("bf16", 40, 2, 256), ("f32", 5, 2, 64),
    ("f32", 40, 2, 128), ("f32", 20, 2, 252)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n", [300, 3000])
def test_infinite_values_of_the_context(n, bad, dtype, T, H, dh):
    """sum p v of an infinite v is infinite wherever the slot stands, and NaN of both signs; the other channels keep
    their bits."""
    lib = need_gpu()
    q, k, v = make(1, T, H, 2, dh, n + T, dtype, T + dh + n)
    ln = torch.tensor([n], dtype=torch.int32).cuda()
    w, w2 = (torch.zeros(1, 2, n + T).cuda() for _ in range(2))
    clean = lib.tree_attention(q, k, v, ln, weights_out=w).float()
    v2 = v.clone()
    v2[:, 17, 0, 3::7] = bad
    v2[:, 150, 0, 4] = float("inf")
    v2[:, 201, 0, 4] = -float("inf")
    got = lib.tree_attention(q, k, v2, ln, weights_out=w2).float()
    G = H // 2
    clean[:, :, :G, 3::7] = bad
    clean[:, :, :G, 4] = float("nan")
    assert same(got, clean)
    assert torch.equal(w, w2)


@pytest.mark.parametrize("dtype,T,dh", [("bf16", 5, 128), ("bf16", 40, 128), ("bf16", 40, 256), ("f32", 5, 64), ("f32", 40, 128)])
@pytest.mark.parametrize("n", [300, 3000])
def test_infinite_values_under_weights_that_vanish(n, dtype, T, dh):
    """exp(s - max) of the slot is below every fp32 number, not 0: its infinite value still counts."""
    lib = need_gpu()
    q, k, v = make(1, T, 2, 2, dh, n + T, dtype, 3)
    q[..., 0] = 1.0
    k[..., 0] = 0.0
    k[:, 230:, :, 0] = 200.0   # scores of 200 and more above those before
    k[:, 17, :, 0] = -200.0
    ln = torch.tensor([n], dtype=torch.int32).cuda()
    clean = lib.tree_attention(q, k, v, ln, scale=1.0).float()
    v2 = v.clone()
    v2[:, 17, 0, 3] = float("inf")
    v2[:, 101, 1, 2] = -float("inf")
    got = lib.tree_attention(q, k, v2, ln, scale=1.0).float()
    clean[:, :, 0, 3] = float("inf")
    clean[:, :, 1, 2] = -float("inf")
    assert same(got, clean)


@pytest.mark.parametrize("T,H,dh,n", [(33, 2, 128, 700), (61, 8, 128, 4100), (150, 2, 64, 1000), (256, 2, 128, 64),
                                      (40, 4, 72, 500), (17, 2, 256, 900), (60, 2, 200, 300)])
def test_many_rows_are_as_exact_as_few(T, H, dh, n):
    """The weights enter the products with 16 significant bits whatever the number of rows: the bar of few rows,
    2^-8 |out| (the output's own rounding) + 1e-4 of the largest."""
    lib = need_gpu()
    q, k, v = make(1, T, H, 2, dh, n + T, "bf16", T + n, spread=1.5)
    parents = trees(1, T, np.random.default_rng(T))
    mask, sees = lib.tree_mask(parents)[0], od.tree_mask(parents)[0]
    out = lib.tree_attention(q, k, v, torch.tensor([n], dtype=torch.int32).cuda(), tree_mask=torch.from_numpy(mask).cuda())
    check(out, od.tree_attention(np64(q), np64(k), np64(v), [n], sees)[0], "bf16")
