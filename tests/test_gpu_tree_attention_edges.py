"""spider_tree_attention at its edges, against the float64 oracle: splits of the keys that a
ceiling leaves without a tile.

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
