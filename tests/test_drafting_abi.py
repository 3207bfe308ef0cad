"""The operators for drafting over the cache without a GPU: the host-only tree mask, and
every refusal, which comes before any HIP call."""
import ctypes
import os

import numpy as np
import pytest

from oracle import drafting as od

lib_mod = pytest.importorskip("paper_2609_34977_amd._lib")
OK, INVALID, SHAPE, UNSUPPORTED, WORKSPACE, HIP = 0, 1, 2, 3, 4, 5
P = 0x100000


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lib_mod._LIB_PATH):
        pytest.skip("libspider.so not built")
    return lib_mod.lib()


@pytest.mark.parametrize("B,T", [(1, 1), (3, 5), (2, 63), (2, 64), (1, 65), (2, 130), (1, 256)])
def test_tree_mask_matches_the_oracle(L, B, T):
    rng = np.random.default_rng(T)
    parents = np.stack([[rng.integers(-1, t) if t else -1 for t in range(T)] for _ in range(B)]).astype(np.int32)
    parents[-1, max(1, T - 3):] = -2
    mask, depth = lib_mod.tree_mask(parents)
    sees, d = od.tree_mask(parents)
    assert np.array_equal(mask, od.pack_mask(sees)) and np.array_equal(depth, d)


def test_tree_mask_by_hand(L):
    mask, depth = lib_mod.tree_mask([[-1, 0, 0, 1, -1, -2]])
    assert mask[0, :, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0]
    assert depth[0].tolist() == [0, 1, 1, 2, 0, 0]


@pytest.mark.parametrize("parents,status", [
    ([[0]], INVALID), ([[-1, 1]], INVALID), ([[-1, 5]], INVALID), ([[-3]], INVALID), ([[-1, -2, 0]], INVALID),
    ([[-2, 0]], INVALID), ([[-1] * 257], UNSUPPORTED)])
def test_tree_mask_refusals(L, parents, status):
    with pytest.raises(lib_mod.SpiderError) as e:
        lib_mod.tree_mask(parents)
    assert e.value.status == status
    assert L.spider_tree_mask(1, 1, None, P, None) == INVALID
    assert L.spider_tree_mask(0, 1, P, P, None) == INVALID


def tree(L, **kw):
    a = dict(B=2, T=3, H=4, Hkv=2, dh=64, q=P, qb=768, qt=256, k=P, v=P, kb=12800, ks=128, kh=64, cap=100, lens=P,
             nodes=None, mask=None, dt=1, scale=0.125, out=P, wi=None, wo=None, ws=P, wsb=1 << 30)
    a.update(kw)
    return L.spider_tree_attention(*a.values(), None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(q=None), INVALID, b"null"), (dict(k=None), INVALID, b"null"), (dict(v=None), INVALID, b"null"),
    (dict(lens=None), INVALID, b"null"), (dict(out=None), INVALID, b"null"), (dict(dt=2), INVALID, b"dtype"),
    (dict(wi=P), INVALID, b"weights_in"), (dict(B=0), INVALID, b"positive"), (dict(T=0), INVALID, b"positive"),
    (dict(cap=0), INVALID, b"positive"), (dict(dh=0), INVALID, b"positive"), (dict(Hkv=0), INVALID, b"positive"),
    (dict(Hkv=3), SHAPE, b"kv heads"), (dict(T=257), UNSUPPORTED, b"T <="), (dict(dh=264), UNSUPPORTED, b"dh <="),
    (dict(B=65536), UNSUPPORTED, b"65535"), (dict(dh=60), UNSUPPORTED, b"16 bytes"),
    (dict(dt=0, dh=6), UNSUPPORTED, b"16 bytes"), (dict(qt=257), INVALID, b"stride"), (dict(ks=129), INVALID, b"stride"),
    (dict(kh=-64), INVALID, b"stride"), (dict(q=P + 2), INVALID, b"aligned"), (dict(v=P + 8), INVALID, b"aligned"),
    (dict(out=P + 4), INVALID, b"aligned"), (dict(wo=P, wsb=8), WORKSPACE, b"workspace"),
    (dict(wo=P, ws=None), WORKSPACE, b"workspace"), (dict(wo=P, ws=P + 16), INVALID, b"256")])
def test_tree_attention_refusals(L, kw, status, word):
    assert tree(L, **kw) == status
    assert word in L.spider_last_error()


def test_tree_attention_workspace_of_bad_sizes_is_zero(L):
    f = L.spider_tree_attention_workspace_size
    assert f(2, 3, 4, 2, 64, 100, 1, 1) > 0
    for bad in ((0, 3, 4, 2, 64, 100, 1), (2, 257, 4, 2, 64, 100, 1), (2, 3, 4, 3, 64, 100, 1), (2, 3, 4, 2, 512, 100, 1),
                (2, 3, 4, 2, 64, 0, 1), (2, 3, 4, 2, 64, 100, 7)):
        assert f(*bad, 1) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(w=None), INVALID), (dict(lens=None), INVALID), (dict(idx=None), INVALID), (dict(new=None), INVALID),
    (dict(L=0), INVALID), (dict(cap=0), INVALID), (dict(keep=0), INVALID), (dict(first=-1), INVALID),
    (dict(last=-1), INVALID), (dict(shared=2), INVALID), (dict(first=6, last=5), SHAPE), (dict(keep=101), SHAPE),
    (dict(first=2147483647, last=2147483647), SHAPE), (dict(L=65536, B=65536), UNSUPPORTED),
    (dict(cap=(1 << 30) + 1), UNSUPPORTED), (dict(cap=20000, wsb=64), WORKSPACE), (dict(cap=20000, ws=None), WORKSPACE), (dict(cap=20000, ws=P + 64), INVALID)])
def test_cache_select_refusals(L, kw, status):
    a = dict(L=2, B=2, Hkv=2, cap=100, w=P, lens=P, keep=10, first=2, last=3, shared=0, idx=P, new=P,
             ws=P, wsb=1 << 30)
    a.update(kw)
    assert L.spider_cache_select(*a.values(), None) == status
    assert b"spider_cache_select" in L.spider_last_error()


def test_cache_select_workspace_of_bad_sizes_is_zero(L):
    f = L.spider_cache_select_workspace_size
    assert f(2, 2, 2, 100, 0) == 0 and f(2, 2, 2, 20000, 0) > f(2, 2, 2, 20000, 1) > 0
    for bad in ((0, 2, 2, 20000, 0), (2, 2, 2, 0, 0), (2, 2, 2, 20000, 2), (65536, 65536, 1, 20000, 0)):
        assert f(*bad) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), INVALID), (dict(vo=None), INVALID), (dict(idx=None), INVALID), (dict(si=None), INVALID),
    (dict(dt=3), INVALID), (dict(L=0), INVALID), (dict(n=-1), INVALID), (dict(il=3), SHAPE), (dict(ih=3), SHAPE),
    (dict(wi=P), INVALID), (dict(wo=P), INVALID), (dict(dh=4), UNSUPPORTED), (dict(dh=264), UNSUPPORTED),
    (dict(k=P + 8), INVALID), (dict(si=(1, 2, 3, 4)), INVALID), (dict(so=(6400, 3200, 32, -16)), INVALID),
    (dict(ko=P), INVALID), (dict(ko=P, vo=2 * P, cap_out=50), SHAPE), (dict(ko=P, vo=2 * P, so=(64, 32, 32, 16)), SHAPE),
    (dict(ko=P, vo=2 * P, wi=P, wo=2 * P), INVALID), (dict(wi=P, wo=P), INVALID), (dict(B=40000), UNSUPPORTED),
    (dict(n=(1 << 25) + 1), UNSUPPORTED)])
def test_cache_compact_refusals(L, kw, status):
    a = dict(L=2, B=2, Hkv=2, dh=16, dt=1, k=P, v=2 * P, si=(6400, 3200, 32, 16), cap=100, ko=3 * P, vo=4 * P,
             so=(6400, 3200, 32, 16), cap_out=100, idx=P, il=1, ih=1, n=5, count=None, base=None, wi=None, wo=None)
    a.update(kw)
    for s in ("si", "so"):
        a[s] = None if a[s] is None else (ctypes.c_int64 * 4)(*a[s])
    assert L.spider_cache_compact(*a.values(), None) == status
    assert b"spider_cache_compact" in L.spider_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(out=None, nxt=None), INVALID), (dict(dt=5), INVALID), (dict(B=0), INVALID),
    (dict(V=0), INVALID), (dict(nb=-1), INVALID), (dict(T=257), UNSUPPORTED), (dict(B=65536), UNSUPPORTED),
    (dict(V=1 << 29), UNSUPPORTED), (dict(nb=32769, bi=P, bv=P), UNSUPPORTED), (dict(h=P), INVALID),
    (dict(h=P, nh=P, hs=-1), INVALID), (dict(h=P, nh=P, hs=1 << 31), INVALID), (dict(nb=3), INVALID),
    (dict(nb=3, bi=P), INVALID), (dict(xs=99), SHAPE), (dict(os=99), SHAPE), (dict(m=P, ms=3), SHAPE),
    (dict(m=P, ms=-4), SHAPE), (dict(out=P, os=120), INVALID), (dict(out=P, dt=1), INVALID), (dict(x=P + 2), INVALID),
    (dict(out=2 * P + 2), INVALID), (dict(V=40000, xs=40000, os=40000, wsb=8), WORKSPACE),
    (dict(V=40000, xs=40000, os=40000, ws=None), WORKSPACE), (dict(V=40000, xs=40000, os=40000, ws=P + 8), INVALID)])
def test_adjust_logits_refusals(L, kw, status):
    a = dict(B=2, T=2, V=100, x=P, xs=100, dt=0, h=None, hs=0, nh=None, np=None, nn=None, tok=None, tree=None, rep=None,
             freq=None, pres=None, bi=None, bv=None, nb=0, m=None, ms=0, out=2 * P, os=100, nxt=P, ws=P, wsb=1 << 20)
    a.update(kw)
    assert L.spider_adjust_logits(*a.values(), None) == status
    assert b"spider_adjust_logits" in L.spider_last_error()


def test_adjust_logits_workspace_of_bad_sizes_is_zero(L):
    f = L.spider_adjust_logits_workspace_size
    assert f(2, 2, 40000) > 0 and f(2, 2, 32768) == 0
    for bad in ((0, 1, 1), (1, 257, 1), (65536, 1, 1), (1, 1, 0), (1, 1, 1 << 29)):
        assert f(*bad) == 0
