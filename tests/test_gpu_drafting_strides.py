"""Layouts that the binding of the operators for drafting takes: the stride of a dimension of
size 1 means nothing and is not looked at."""
import pytest
import torch

from gpu_common import need_gpu

pytestmark = pytest.mark.gpu


def odd(t, dim):
    """t with another stride, no multiple of 16 bytes, in a dimension of size 1."""
    strides = list(t.stride())
    strides[dim] = 7 * strides[dim] + 3
    return t.as_strided(t.shape, strides)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tree_attention_of_one_sample_one_head_or_one_slot(dtype):
    lib = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    for B, T, H, cap in ((1, 3, 2, 40), (2, 1, 1, 40), (2, 1, 1, 1)):
        q, k, v = rand(B, T, H, 64), rand(B, cap, H, 64), rand(B, cap, H, 64)
        ln = torch.full((B,), max(0, cap - T - 3), dtype=torch.int32, device="cuda")
        want = lib.tree_attention(q, k, v, ln)
        dims = [i for i in range(3) if k.shape[i] == 1]
        for i in dims:
            assert torch.equal(lib.tree_attention(q, odd(k, i), v, ln), want)
            assert torch.equal(lib.tree_attention(q, k, odd(v, i), ln), want)
        for i in (i for i in range(3) if q.shape[i] == 1):
            assert torch.equal(lib.tree_attention(odd(q, i), k, v, ln), want)


def test_compact_of_one_layer_one_sample_or_one_head():
    lib = need_gpu()
    for L, B, Hkv in ((1, 2, 2), (2, 1, 2), (2, 2, 1), (1, 1, 1)):
        k, v = torch.randn(L, B, 20, Hkv, 16, device="cuda"), torch.randn(L, B, 20, Hkv, 16, device="cuda")
        idx = torch.tensor([2, 5, 11], dtype=torch.int32, device="cuda").expand(1, B, 1, 3).contiguous()
        for i in (i for i in (0, 1, 3) if k.shape[i] == 1):
            for inplace in (False, True):
                k1, v1, k2, v2 = k.clone(), v.clone(), k.clone(), v.clone()
                kw = {} if inplace else dict(k_out=odd(k2, i), v_out=v2)
                lib.cache_compact(odd(k1, i), v1, idx, **kw)
                for src, dst in ((k, k1 if inplace else k2), (v, v1 if inplace else v2)):
                    assert torch.equal(dst[:, :, :3], src[:, :, [2, 5, 11]]) and torch.equal(dst[:, :, 3:], src[:, :, 3:])
