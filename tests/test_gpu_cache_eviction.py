"""spider_cache_select and spider_cache_compact against the oracle: indices, lengths and
moved rows are equal, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import drafting as od
from gpu_common import need_gpu

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def weights(kind, shape, rng):
    w = rng.exponential(1.0, shape).astype(np.float32) ** 3
    if kind == "ties":
        w = np.floor(4 * w).astype(np.float32)
    elif kind == "zeros":
        w[rng.random(shape) < 0.9] = 0.0
        w[rng.random(shape) < 0.1] = -0.0
    elif kind == "odd":
        w[rng.random(shape) < 0.1] = np.nan
        w[rng.random(shape) < 0.1] = np.inf
        w[rng.random(shape) < 0.1] = -np.inf
        w[rng.random(shape) < 0.1] *= -1
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "tiny":
        w *= np.float32(1e-42)  # subnormal
    return w


@pytest.mark.parametrize("kind", ["plain", "ties", "zeros", "odd", "equal", "tiny"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("shape,lens,keep,first,last", [
    ((2, 3, 4, 333), [333, 222, 50], 100, 4, 32),
    ((1, 2, 1, 70), [70, 0], 1, 0, 0),
    ((1, 3, 2, 1030), [1025, 1024, 1023], 1023, 1, 1),
    ((1, 1, 3, 2050), [2050], 700, 0, 700),
    ((1, 1, 2, 5000), [4999], 4998, 2, 0),
    ((1, 2, 2, 9), [9, -3], 9, 0, 0),
    ((2, 1, 1, 20000), [20000], 1234, 10, 20),
    ((1, 3, 2, 16385), [16385, 16384, 8193], 8192, 3, 5),
    ((1, 2, 3, 8200), [8193, 8192], 8000, 0, 7999),
    ((2, 2, 2, 24600), [24577, 40], 24576, 0, 1),
    ((1, 1, 300, 33000), [30001], 77, 1, 1),
])
def test_select(kind, shared, shape, lens, keep, first, last):
    lib = need_gpu()
    w = weights(kind, shape, np.random.default_rng(keep))
    idx, new = lib.cache_select(torch.from_numpy(w).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), keep,
                                n_first=first, n_last=last, shared=shared)
    with np.errstate(invalid="ignore"):
        ref, rnew = od.cache_select(w, lens, keep, first, last, shared)
    assert np.array_equal(new.cpu().numpy(), rnew)
    assert np.array_equal(idx.cpu().numpy(), ref)


@pytest.mark.parametrize("keep", [1, 5000, 65537, 199000])
def test_select_from_a_long_cache(keep):
    lib = need_gpu()
    w = torch.empty(1, 2, 2, 200000, device="cuda").exponential_(generator=torch.Generator(device="cuda").manual_seed(3))
    w = torch.floor(w * 50) / 50
    lens = torch.tensor([200000, 131072], dtype=torch.int32).cuda()
    idx, new = lib.cache_select(w, lens, keep, n_first=min(4, keep - 1), n_last=keep // 4)
    ref, rnew = od.cache_select(w.cpu().numpy(), [200000, 131072], keep, min(4, keep - 1), keep // 4)
    assert np.array_equal(new.cpu().numpy(), rnew) and np.array_equal(idx.cpu().numpy(), ref)


def test_select_from_many_long_rows():
    lib = need_gpu()
    w = weights("ties", (1, 1, 30, 66000), np.random.default_rng(8))
    idx, new = lib.cache_select(torch.from_numpy(w).cuda(), torch.tensor([20001], dtype=torch.int32).cuda(), 6000, n_last=50)
    ref, rnew = od.cache_select(w, [20001], 6000, 0, 50)
    assert np.array_equal(new.cpu().numpy(), rnew) and np.array_equal(idx.cpu().numpy(), ref)


def caches(L, B, cap, Hkv, dh, dtype, heads_first, seed):
    g = torch.Generator().manual_seed(seed)
    shape = (L, B, Hkv, cap, dh) if heads_first else (L, B, cap, Hkv, dh)
    t = [torch.randn(shape, generator=g).to(DT[dtype]).cuda() for _ in range(2)]
    return [x.transpose(2, 3) for x in t] if heads_first else t


@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("L,B,cap,Hkv,dh,dtype,heads_first,shared,layers", [
    (2, 3, 333, 4, 32, "f32", False, True, True),
    (2, 2, 700, 3, 128, "bf16", False, False, True),
    (1, 2, 301, 2, 80, "bf16", True, False, True),
    (3, 1, 90, 2, 256, "f32", True, True, False),
    (2, 2, 1500, 2, 8, "bf16", False, False, False),
    (1, 1, 2500, 1, 4, "f32", False, False, True),
])
def test_compact(inplace, L, B, cap, Hkv, dh, dtype, heads_first, shared, layers):
    lib = need_gpu()
    rng = np.random.default_rng(cap)
    k, v = caches(L, B, cap, Hkv, dh, dtype, heads_first, 1)
    n = cap // 2
    # ascending slots; some rows start with a run that stays where it is
    idx = np.stack([np.sort(rng.permutation(cap)[:n]) for _ in range((L if layers else 1) * B * (1 if shared else Hkv))])
    idx[::2, :n // 3] = np.arange(n // 3)
    idx[::2, n // 3:] = n // 3 + 1 + np.sort(rng.permutation(cap - n // 3 - 1)[:n - n // 3])
    idx = idx.reshape(L if layers else 1, B, 1 if shared else Hkv, n).astype(np.int32)
    count = np.array([n - 5 * b for b in range(B)], np.int32)
    w = torch.from_numpy(rng.random((L, B, Hkv, cap)).astype(np.float32)).cuda()
    cap_out = cap if inplace else n + 3
    if inplace:
        k_out, v_out, w_out = k, v, w
    else:
        k_out, v_out = caches(L, B, cap_out, Hkv, dh, dtype, not heads_first, 2)
        w_out = torch.rand(L, B, Hkv, cap_out).cuda()
    np32 = lambda t: t.float().cpu().numpy()  # noqa: E731
    want = [od.cache_compact(np32(a), np32(o), idx, count) for a, o in ((k, k_out), (v, v_out))]
    ww = od.cache_compact(np32(w).transpose(0, 1, 3, 2), np32(w_out).transpose(0, 1, 3, 2), idx, count).transpose(0, 1, 3, 2)
    kw = {} if inplace else dict(k_out=k_out, v_out=v_out, weights_out=w_out)
    lib.cache_compact(k, v, torch.from_numpy(idx).cuda(), torch.from_numpy(count).cuda(), weights=w, **kw)
    assert np.array_equal(np32(k_out), want[0]) and np.array_equal(np32(v_out), want[1])
    assert np.array_equal(np32(w_out), ww)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accepted_nodes_move_behind_their_context(dtype):
    lib = need_gpu()
    L, B, cap, Hkv, dh = 3, 3, 64, 2, 64
    k, v = caches(L, B, cap, Hkv, dh, dtype, False, 4)
    base = np.array([40, 0, 62], np.int32)
    idx = np.array([[0, 2, 5, 9], [1, 2, 3, 4], [1, 2, 3, 4]], np.int32).reshape(1, B, 1, 4)  # the last runs off the cache
    count = np.array([4, 3, 4], np.int32)
    np32 = lambda t: t.float().cpu().numpy()  # noqa: E731
    want = [od.cache_compact(np32(x), np32(x), idx, count, base) for x in (k, v)]
    lib.cache_compact(k, v, *(torch.from_numpy(x).cuda() for x in (idx, count)), base=torch.from_numpy(base).cuda())
    assert np.array_equal(np32(k), want[0]) and np.array_equal(np32(v), want[1])


def test_entries_outside_the_caches_move_nothing():
    lib = need_gpu()
    k, v = caches(1, 2, 30, 2, 16, "bf16", False, 5)
    k_out, v_out = caches(1, 2, 4, 2, 16, "bf16", False, 6)
    idx = np.array([[-1, 29, 30, 5, 6, 7], [2000000000, -7, 3, 4, 0, 1]], np.int32).reshape(1, 2, 1, 6)
    base = np.array([0, -1], np.int32)
    np32 = lambda t: t.float().cpu().numpy()  # noqa: E731
    want = [od.cache_compact(np32(a), np32(o), idx, None, base) for a, o in ((k, k_out), (v, v_out))]
    lib.cache_compact(k, v, torch.from_numpy(idx).cuda(), base=torch.from_numpy(base).cuda(), k_out=k_out, v_out=v_out)
    assert np.array_equal(np32(k_out), want[0]) and np.array_equal(np32(v_out), want[1])
    empty = torch.empty(1, 2, 1, 0, dtype=torch.int32).cuda()
    before = k.clone()
    lib.cache_compact(k, v, empty)
    assert torch.equal(k, before)


def test_a_cache_past_four_gigabytes():
    lib = need_gpu()
    L, B, cap, Hkv, dh = 2, 1, 300000, 32, 128
    k = torch.zeros(L, B, cap, Hkv, dh, dtype=torch.bfloat16, device="cuda")
    k[:] = torch.arange(cap, device="cuda", dtype=torch.float32).remainder(251).bfloat16()[None, None, :, None, None]
    v = -k
    idx = torch.arange(100, dtype=torch.int32, device="cuda").mul(2999).add(3).view(1, 1, 1, 100)
    want = k[:, :, idx.view(-1).long()].clone()
    lib.cache_compact(k, v, idx)
    assert torch.equal(k[:, :, :100], want) and torch.equal(v[:, :, :100], -want)


def test_captured():
    lib = need_gpu()
    L, B, cap, Hkv, dh = 2, 2, 400, 2, 64
    k, v = caches(L, B, cap, Hkv, dh, "bf16", False, 7)
    k0, v0 = k.clone(), v.clone()
    w = torch.rand(L, B, Hkv, cap).cuda()
    w0 = w.clone()
    lens = torch.tensor([400, 300], dtype=torch.int32).cuda()
    lib.cache_select(w, lens, 100)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        idx, new = lib.cache_select(w, lens, 100, n_first=2, n_last=9)
        lib.cache_compact(k, v, idx, new, weights=w)
    for i in range(3):
        w0 = torch.roll(w0, 17, 3)
        w.copy_(w0), k.copy_(k0), v.copy_(v0)
        graph.replay()
        torch.cuda.synchronize()
        i2, n2 = lib.cache_select(w0, lens, 100, n_first=2, n_last=9)
        k2, v2, w2 = k0.clone(), v0.clone(), w0.clone()
        lib.cache_compact(k2, v2, i2, n2, weights=w2)
        assert torch.equal(idx, i2) and torch.equal(k, k2) and torch.equal(v, v2) and torch.equal(w, w2)


def test_refusals_of_the_binding():
    lib = need_gpu()
    k, v = caches(2, 2, 30, 2, 16, "bf16", False, 8)
    k_out, v_out = caches(2, 2, 30, 2, 16, "bf16", False, 9)
    idx = torch.zeros(1, 2, 1, 3, dtype=torch.int32).cuda()
    w = torch.zeros(2, 2, 2, 30).cuda()
    lens = torch.tensor([3, 3], dtype=torch.int32).cuda()
    bad = [
        lambda: lib.cache_compact(k, v, idx.long()),
        lambda: lib.cache_compact(k, v, idx[:, :1]),
        lambda: lib.cache_compact(k, v, idx.expand(3, 2, 1, 3).contiguous()),
        lambda: lib.cache_compact(k, v, idx, k_out=k_out),
        lambda: lib.cache_compact(k, v, idx, k_out=k_out, v_out=v_out, weights=w),
        lambda: lib.cache_compact(k, v, idx, k_out=k, v_out=v_out),
        lambda: lib.cache_compact(k, v, idx, k_out=k_out.float(), v_out=v_out.float()),
        lambda: lib.cache_compact(k, v[:, :, ::2], idx),
        lambda: lib.cache_compact(k[..., :4], v[..., :4], idx),
        lambda: lib.cache_select(w, lens, 31),
        lambda: lib.cache_select(w, lens, 0),
        lambda: lib.cache_select(w, lens, 5, n_first=3, n_last=3),
        lambda: lib.cache_select(w, lens, 5, n_first=-1),
        lambda: lib.cache_select(w.double(), lens, 5),
        lambda: lib.cache_select(w, lens.long(), 5),
    ]
    for f in bad:
        with pytest.raises((ValueError, TypeError, lib.SpiderError)):
            f()


@pytest.mark.parametrize("L,B,cap,Hkv,dh,keep", [(2, 2, 3000, 4, 128, 2500), (1, 1, 9000, 2, 64, 8900)])
def test_in_place_over_many_pieces(L, B, cap, Hkv, dh, keep):
    """Thousands of entries that move a little: every piece's reads come before its writes."""
    lib = need_gpu()
    k, v = caches(L, B, cap, Hkv, dh, "bf16", False, 12)
    w = torch.rand(L, B, Hkv, cap).cuda()
    lens = torch.full((B,), cap, dtype=torch.int32).cuda()
    idx, new = lib.cache_select(w, lens, keep)
    at = idx.long().transpose(2, 3)
    want = [torch.gather(x, 2, at[..., None].expand(-1, -1, -1, -1, dh)) for x in (k, v)]
    ww = torch.gather(w, 3, idx.long())
    tail = k[:, :, keep:].clone()
    lib.cache_compact(k, v, idx, new, weights=w)
    assert torch.equal(k[:, :, :keep], want[0]) and torch.equal(v[:, :, :keep], want[1])
    assert torch.equal(w[..., :keep], ww) and torch.equal(k[:, :, keep:], tail)
