"""spider_adjust_logits: bias lists that name some tokens several times, compared bit for bit
with the entries added one after the other in fp32."""
import numpy as np
import pytest
import torch

from gpu_common import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,nb", [(500, 300), (32000, 1500), (40000, 4001), (9000, 32768), (70001, 32768)])
def test_bias_entries_of_a_token_add_up_in_order(V, nb):
    """Tokens with one entry, with two and with many, side by side in every piece of the vocabulary."""
    lib = need_gpu()
    rng = np.random.default_rng(nb)
    x = rng.normal(0, 3, (2, V)).astype(np.float32)
    ids = np.where(rng.random((2, nb)) < 0.7, rng.integers(0, V, (2, nb)), rng.integers(0, max(2, V // 50), (2, nb)) * 40 % V)
    ids[:, 5] = ids[:, 2] = ids[:, nb - 1]
    ids[1, :] = np.where(np.arange(nb) % 7 == 3, -1, ids[1])
    ids = ids.astype(np.int32)
    bias = rng.normal(0, 5, (2, nb)).astype(np.float32)
    want = x.copy()
    for b in range(2):
        add = np.zeros(V, np.float32)
        for v, w in zip(ids[b], bias[b]):
            if v >= 0:
                add[v] = add[v] + w
        want[b] += add
    out, nxt = lib.adjust_logits(torch.from_numpy(x).cuda(), bias_ids=torch.from_numpy(ids).cuda(), bias=torch.from_numpy(bias).cuda())
    assert np.array_equal(out.cpu().numpy(), want)
    assert np.array_equal(nxt.cpu().numpy(), want.argmax(1))
