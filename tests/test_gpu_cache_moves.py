"""spider_cache_compact in place over many streams (256 and more: columns of 128 bytes), every
layer of a cache at once: equal, bit for bit."""
import pytest
import torch

from gpu_common import need_gpu
from test_gpu_cache_eviction import DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L,B,cap,Hkv,dh,dtype,keep", [
    (32, 1, 1500, 32, 128, "bf16", 700), (4, 2, 3000, 32, 128, "bf16", 2900), (8, 4, 600, 8, 80, "bf16", 333),
    (16, 16, 90, 1, 8, "bf16", 45), (4, 8, 700, 8, 256, "f32", 512), (2, 32, 400, 4, 36, "f32", 399)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_in_place_over_many_streams(heads_first, L, B, cap, Hkv, dh, dtype, keep):
    lib = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(cap)
    shape = (L, B, Hkv, cap, dh) if heads_first else (L, B, cap, Hkv, dh)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    if heads_first:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    w = torch.rand(L, B, Hkv, cap, generator=g, device="cuda")
    idx = torch.argsort(torch.rand(L, B, Hkv, cap, generator=g, device="cuda"), -1)[..., :keep].sort(-1).values
    count = torch.tensor([keep - 7 * b for b in range(B)], dtype=torch.int32).clamp(min=0).cuda()
    on = torch.arange(keep, device="cuda")[None] < count[:, None]
    at = idx.transpose(2, 3)[..., None].expand(-1, -1, -1, -1, dh)
    want = []
    for x in (k, v):
        y = x.clone()
        y[:, :, :keep] = torch.where(on[None, :, :, None, None], torch.gather(x, 2, at), x[:, :, :keep])
        want.append(y)
    ww = w.clone()
    ww[..., :keep] = torch.where(on[None, :, None], torch.gather(w, 3, idx), w[..., :keep])
    lib.cache_compact(k, v, idx.int().contiguous(), count, weights=w)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and torch.equal(w, ww)
