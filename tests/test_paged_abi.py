"""The operators over a paged cache without a GPU: host-only rope_axes, workspace sizes, and refusals before any HIP call."""
import ctypes
import os

import numpy as np
import pytest

from oracle import paged as op

lib_mod = pytest.importorskip("paper_2609_34977_amd._lib")
OK, INVALID, SHAPE, UNSUPPORTED, WORKSPACE, HIP = 0, 1, 2, 3, 4, 5
P = 0x100000


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lib_mod._LIB_PATH):
        pytest.skip("libspider.so not built")
    return lib_mod.lib()


def cache(**kw):
    """A descriptor whose pointers are never followed."""
    a = dict(k=P, v=2 * P, stride_page=16 * 2 * 64, stride_slot=2 * 64, stride_head=64, n_pages=10, page_size=16, table=3 * P, table_stride=8,
             max_pages=8, lens=4 * P, cu=5 * P, B=3)
    a.update(kw)
    return lib_mod.PagedCache(*a.values())


BAD_CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(cu=None), INVALID),
    (dict(B=0), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(B=65536), UNSUPPORTED),
    (dict(page_size=0), UNSUPPORTED), (dict(page_size=4), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED),
    (dict(max_pages=(1 << 26) + 1, table_stride=1 << 27), UNSUPPORTED), (dict(table_stride=7), SHAPE),
    (dict(stride_page=-2048), INVALID), (dict(stride_slot=129), INVALID), (dict(stride_head=60), INVALID), (dict(k=P + 8), INVALID), (dict(v=2 * P + 2), INVALID),
]


@pytest.mark.parametrize("rot,sections,inter", [
    (128, [64], False), (128, [64], True), (128, [16, 24, 24], False), (128, [24, 20, 20], True), (40, [8, 6, 6], True), (80, [10] * 4, True),
    (80, [0, 40, 0], False), (6, [1, 1, 1], True), (6, [3, 0, 0], True), (2, [1], False), (256, [16] * 8, True),
])
def test_rope_axes_matches_oracle(rot, sections, inter):
    freq, axis = lib_mod.rope_axes(rot, 10000.0, sections, inter)
    want = op.rope_axes(rot, 10000.0, sections, inter)
    assert np.array_equal(axis, want[1])
    assert np.allclose(freq, want[0], rtol=1e-14, atol=0)


@pytest.mark.parametrize("change,status", [
    (dict(rot=0), INVALID), (dict(rot=63), INVALID), (dict(rot=258), UNSUPPORTED), (dict(theta=0.0), INVALID), (dict(theta=float("inf")), INVALID),
    (dict(theta=float("nan")), INVALID), (dict(n=0), INVALID), (dict(n=9), UNSUPPORTED), (dict(sections=[16, 8, 9]), SHAPE), (dict(sections=[16, 17, -1]), INVALID),
    (dict(sections=[8, 12, 12], inter=1), SHAPE), (dict(inter=2), INVALID), (dict(freq=None), INVALID), (dict(axis=None), INVALID),
])
def test_rope_axes_refusals(L, change, status):
    a = dict(rot=64, theta=1e4, n=3, sections=[16, 8, 8], inter=0, freq=np.zeros(128), axis=np.zeros(128, np.uint8))
    a.update(change)
    s = np.array(list(a["sections"]) + [0] * 8, np.int32)
    ptr = lambda x: None if x is None else x.ctypes.data
    assert L.spider_rope_axes(a["rot"], a["theta"], a["n"], s.ctypes.data, a["inter"], ptr(a["freq"]), ptr(a["axis"])) == status
    assert b"spider_rope_axes" in L.spider_last_error()


ROPE = dict(N=9, H=4, Hkv=2, dh=64, rot=64, axes=3, pos=6 * P, ps=9, freq=7 * P, axis=8 * P, q=9 * P, qs=256, qo=10 * P, qos=256, k=11 * P, ks=128,
            v=12 * P, vs=128, cache=None, dt=1)


@pytest.mark.parametrize("change,status", [
    (dict(pos=None), INVALID), (dict(freq=None), INVALID), (dict(axis=None), INVALID), (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(q=None, qo=None, k=None, v=None, cache=0), INVALID), (dict(cache=0), INVALID), (dict(dt=2), INVALID), (dict(N=0), INVALID),
    (dict(N=1 << 24), UNSUPPORTED), (dict(H=0), INVALID), (dict(Hkv=0), INVALID), (dict(axes=0), INVALID), (dict(axes=9), UNSUPPORTED), (dict(dh=60), UNSUPPORTED),
    (dict(dh=264, rot=64), UNSUPPORTED), (dict(rot=0), SHAPE), (dict(rot=63), SHAPE), (dict(rot=66), SHAPE), (dict(ps=8), SHAPE), (dict(qs=252), INVALID),
    (dict(qs=248), INVALID), (dict(ks=120), INVALID), (dict(vs=0), INVALID), (dict(q=9 * P + 4), INVALID), (dict(qo=9 * P, qos=512), INVALID),
])
def test_rope_append_refusals(L, change, status):
    a = dict(ROPE, cache=cache())
    a.update(change)
    a["cache"] = ctypes.byref(a["cache"]) if a["cache"] else None
    assert L.spider_rope_append(*a.values(), None) == status
    assert b"spider_rope_append" in L.spider_last_error()


@pytest.mark.parametrize("change,status", BAD_CACHES + [(dict(stride_slot=0), INVALID), (dict(stride_page=0), INVALID), (dict(stride_head=0), INVALID)])
def test_rope_append_refuses_caches(L, change, status):
    a = dict(ROPE, cache=ctypes.byref(cache(**change)))
    assert L.spider_rope_append(*a.values(), None) == status
    assert b"spider_rope_append" in L.spider_last_error()


ATTN = dict(N=9, H=4, Hkv=2, dh=64, q=6 * P, qs=256, cache=None, dt=1, scale=0.1, window=0, out=7 * P, ws=8 * P, wsb=1 << 40)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(cache=0), INVALID), (dict(dt=3), INVALID), (dict(N=0), INVALID), (dict(H=0), INVALID), (dict(H=5), SHAPE),
    (dict(window=-1), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(N=1 << 22), UNSUPPORTED), (dict(dh=60), UNSUPPORTED),
    (dict(dh=264), UNSUPPORTED), (dict(qs=252), INVALID), (dict(qs=-256), INVALID), (dict(q=6 * P + 8), INVALID), (dict(out=7 * P + 4), INVALID),
    (dict(ws=None), WORKSPACE), (dict(wsb=255), WORKSPACE), (dict(ws=8 * P + 16), INVALID), (dict(dt=0, dh=2), UNSUPPORTED),
])
def test_paged_attention_refusals(L, change, status):
    a = dict(ATTN, cache=cache(max_pages=800, table_stride=800))
    a.update(change)
    a["cache"] = ctypes.byref(a["cache"]) if a["cache"] else None
    assert L.spider_paged_attention(*a.values(), None) == status
    assert b"spider_paged_attention" in L.spider_last_error()


@pytest.mark.parametrize("change,status", BAD_CACHES + [(dict(B=65535), UNSUPPORTED)])
def test_paged_attention_refuses_caches(L, change, status):
    a = dict(ATTN, cache=ctypes.byref(cache(**change)))
    if change.get("B") == 65535:
        a.update(Hkv=65, H=65)
    assert L.spider_paged_attention(*a.values(), None) == status


FORK = dict(L=2, Hkv=2, dh=64, dt=1, k=P, v=2 * P, st=None, n_pages=10, page=16, M=8, B_in=3, table=3 * P, lens=4 * P, ref=5 * P, B=5, parent=6 * P, new=7 * P,
            t_out=8 * P, l_out=9 * P, r_out=10 * P, missing=11 * P, ws=12 * P, wsb=1 << 30)


@pytest.mark.parametrize("change,status", [(dict([(n, None)]), INVALID) for n in ("k", "v", "table", "lens", "ref", "parent", "t_out", "l_out", "r_out", "missing")] + [
    (dict(dt=2), INVALID), (dict(L=0), INVALID), (dict(n_pages=0), INVALID), (dict(M=0), INVALID), (dict(B_in=0), INVALID), (dict(B=0), INVALID),
    (dict(B=4097), UNSUPPORTED), (dict(B_in=4097), UNSUPPORTED), (dict(L=16384, B=4), UNSUPPORTED), (dict(page=4), UNSUPPORTED), (dict(page=48), UNSUPPORTED),
    (dict(page=8192), UNSUPPORTED), (dict(M=(1 << 26) + 1), UNSUPPORTED), (dict(B=1024, M=1 << 21), UNSUPPORTED), (dict(B_in=1024, M=1 << 21), UNSUPPORTED), (dict(dh=60), UNSUPPORTED), (dict(dh=264), UNSUPPORTED), (dict(Hkv=65536), UNSUPPORTED),
    (dict(k=P + 8), INVALID), (dict(ws=None), WORKSPACE), (dict(wsb=10), WORKSPACE), (dict(ws=12 * P + 128), INVALID),
    (dict(st=[8192, 2048, 128, 60]), INVALID), (dict(st=[0, 2048, 128, 64]), INVALID), (dict(st=[8192, 0, 128, 64]), INVALID), (dict(st=[8192, 2048, 0, 64]), INVALID),
    (dict(st=[8192, 2048, 128, 0]), INVALID), (dict(st=[8192, -2048, 128, 64]), INVALID),
    (dict(t_out=3 * P), INVALID), (dict(t_out=3 * P + 4 * 23), INVALID), (dict(l_out=4 * P + 8), INVALID), (dict(r_out=5 * P), INVALID), (dict(l_out=6 * P), INVALID),
    (dict(missing=7 * P + 16), INVALID), (dict(l_out=8 * P + 4 * 39), INVALID), (dict(missing=10 * P), INVALID),
])
def test_pages_fork_refusals(L, change, status):
    a = dict(FORK, st=[80 * 2048, 2048, 128, 64])
    a.update(change)
    a["st"] = (ctypes.c_int64 * 4)(*a["st"])
    assert L.spider_pages_fork(*a.values(), None) == status
    assert b"spider_pages_fork" in L.spider_last_error()


BEAM = dict(B=2, K=3, M=4, V=100, x=P, xs=100, dt=0, scores=2 * P, done=3 * P, eos=2, s_out=4 * P, p_out=5 * P, t_out=6 * P, d_out=7 * P, h=8 * P, hs=50, nh=9 * P,
            cap=50, h_out=10 * P, hos=50, nh_out=11 * P, ws=12 * P, wsb=1 << 30)


@pytest.mark.parametrize("change,status", [(dict([(n, None)]), INVALID) for n in ("x", "scores", "s_out", "p_out", "t_out", "d_out", "h", "nh", "h_out", "nh_out")] + [
    (dict(dt=2), INVALID), (dict(B=0), INVALID), (dict(K=0), INVALID), (dict(M=0), INVALID), (dict(V=0), INVALID), (dict(K=65), UNSUPPORTED), (dict(M=65), UNSUPPORTED),
    (dict(V=(1 << 19) + 1, xs=1 << 20), UNSUPPORTED), (dict(B=30000), UNSUPPORTED), (dict(xs=99), SHAPE), (dict(eos=100), INVALID), (dict(eos=-2), INVALID),
    (dict(eos=-1), INVALID), (dict(x=P + 2), INVALID), (dict(cap=0), INVALID), (dict(hs=49), SHAPE), (dict(hos=49), SHAPE), (dict(cap=(1 << 24) + 1, hs=1 << 25, hos=1 << 25), SHAPE),
    (dict(ws=None), WORKSPACE), (dict(wsb=100), WORKSPACE), (dict(ws=12 * P + 8), INVALID), (dict(s_out=2 * P), INVALID), (dict(d_out=3 * P + 20), INVALID),
    (dict(nh_out=9 * P), INVALID), (dict(h_out=8 * P), INVALID), (dict(h_out=8 * P + 4 * 299), INVALID),
    (dict(s_out=P + 4 * 599), INVALID), (dict(t_out=8 * P + 4 * 290), INVALID), (dict(t_out=5 * P + 28), INVALID), (dict(h_out=7 * P - 4), INVALID),
    (dict(h_out=3 * P), INVALID), (dict(nh_out=4 * P - 28), INVALID),
])
def test_beam_select_refusals(L, change, status):
    a = dict(BEAM)
    a.update(change)
    assert L.spider_beam_select(*a.values(), None) == status
    assert b"spider_beam_select" in L.spider_last_error()


def test_workspace_sizes(L):
    assert L.spider_paged_attention_workspace_size(0, 1, 4, 2, 64, 9000, 1) == 0
    assert L.spider_paged_attention_workspace_size(9, 3, 5, 2, 64, 9000, 1) == 0
    assert L.spider_paged_attention_workspace_size(1, 1, 4, 2, 64, 0, 1) == 0
    assert L.spider_paged_attention_workspace_size(1, 1, 4, 2, 64, 100, 1) == 0 < L.spider_paged_attention_workspace_size(1, 1, 4, 2, 64, 9000, 1)
    assert L.spider_pages_fork_workspace_size(0, 10) == 0 and L.spider_pages_fork_workspace_size(4097, 10) == 0
    assert L.spider_pages_fork_workspace_size(5, 1000) >= 5 * 16 + 4000
    assert L.spider_beam_select_workspace_size(1, 65, 1, 100) == 0 and L.spider_beam_select_workspace_size(1, 1, 1, (1 << 19) + 1) == 0
    assert L.spider_beam_select_workspace_size(2, 3, 4, 20000) >= 2 * 3 * 3 * (4 * 8 + 12)
