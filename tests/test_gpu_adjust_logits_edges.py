"""spider_adjust_logits: bias lists that name some tokens several times, compared bit for bit
with the entries added one after the other in fp32; the shapes that the binding takes."""
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


def test_a_mask_row_per_sample_for_one_node():
    """[B, W32] masks for T = 1, with logits [B, V] and [B, 1, V]."""
    lib = need_gpu()
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.normal(0, 1, (3, 100)).astype(np.float32)).cuda()
    bits = torch.from_numpy(rng.integers(-2**31, 2**31, (3, 4)).astype(np.int32)).cuda()
    want, ids = lib.adjust_logits(x, mask=bits)
    got, ids1 = lib.adjust_logits(x.unsqueeze(1), mask=bits)
    full, ids2 = lib.adjust_logits(x.unsqueeze(1), mask=bits.unsqueeze(1))
    allowed = (bits.cpu().numpy()[:, np.arange(100) // 32] >> (np.arange(100) % 32)) & 1 == 1
    assert np.array_equal(want.cpu().numpy(), np.where(allowed, x.cpu().numpy(), -np.inf))
    assert torch.equal(got[:, 0], want) and torch.equal(full, got)
    assert torch.equal(ids1[:, 0], ids) and torch.equal(ids2, ids1)
    with pytest.raises(ValueError):
        lib.adjust_logits(torch.zeros(3, 2, 100).cuda(), mask=bits)


def test_a_workspace_of_the_size_that_the_library_names():
    lib = need_gpu()
    for V in (100, 40000):
        x = torch.randn(3, V, device="cuda")
        n = lib.lib().spider_adjust_logits_workspace_size(3, 1, V)
        want, ids = lib.adjust_logits(x)
        for ws in (torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n + 300, dtype=torch.uint8, device="cuda")[44:]):
            got, ids2 = lib.adjust_logits(x, workspace=ws)
            assert torch.equal(got, want) and torch.equal(ids2, ids)
    for ws in (torch.empty(n - 1, dtype=torch.uint8, device="cuda"), torch.empty(n + 40, dtype=torch.uint8, device="cuda")[1:],
               torch.empty(n, dtype=torch.uint8), torch.empty(2 * n + 512, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            lib.adjust_logits(x, workspace=ws)
    with pytest.raises(ValueError):
        lib.adjust_logits(x, bias_ids=torch.zeros(4, dtype=torch.int32, device="cuda"), bias=torch.zeros(4, device="cuda"))
