"""Refusals of the operators for drafting over the cache at the ends of their ranges, before
any HIP call."""
import ctypes
import os

import pytest

lib_mod = pytest.importorskip("paper_2609_34977_amd._lib")
OK, INVALID, SHAPE, UNSUPPORTED, WORKSPACE, HIP = 0, 1, 2, 3, 4, 5
P = 0x100000


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lib_mod._LIB_PATH):
        pytest.skip("libspider.so not built")
    return lib_mod.lib()


@pytest.mark.parametrize("stride", [(1 << 31) - 1, (1 << 31) - (1 << 14) + 1])
def test_adjust_logits_refuses_histories_whose_index_passes_31_bits(L, stride):
    """The index of a history entry runs 8192 past the last one and a count must stay below its flag bit."""
    a = dict(B=2, T=2, V=100, x=P, xs=100, dt=0, h=P, hs=stride, nh=P, np=None, nn=None, tok=None, tree=None, rep=None,
             freq=None, pres=None, bi=None, bv=None, nb=0, m=None, ms=0, out=2 * P, os=100, nxt=P, ws=P, wsb=1 << 20)
    assert L.spider_adjust_logits(*a.values(), None) == INVALID
    assert b"history" in L.spider_last_error()


@pytest.mark.parametrize("new", [P, P + 4, P - 12])
def test_cache_select_refuses_new_lengths_over_the_old_ones(L, new):
    """Rows of a sample read its length while another one writes the new length."""
    a = dict(L=2, B=4, Hkv=2, cap=100, w=2 * P, lens=P, keep=10, first=2, last=3, shared=0, idx=3 * P, new=new, ws=P, wsb=1 << 30)
    assert L.spider_cache_select(*a.values(), None) == INVALID
    assert b"overlap" in L.spider_last_error()


@pytest.mark.parametrize("dim", range(4))
@pytest.mark.parametrize("inplace", [False, True])
def test_cache_compact_refuses_outputs_that_share_memory(L, inplace, dim):
    """A broadcast cache: rows of other layers, samples or heads would be moved over each other."""
    strides = [6400, 3200, 32, 16]
    strides[dim] = 0
    s = (ctypes.c_int64 * 4)(*strides)
    a = dict(L=2, B=2, Hkv=2, dh=16, dt=1, k=P, v=2 * P, si=s, cap=100, ko=P if inplace else 3 * P,
             vo=2 * P if inplace else 4 * P, so=s, cap_out=100, idx=P, il=1, ih=1, n=5, count=None, base=None, wi=None, wo=None)
    assert L.spider_cache_compact(*a.values(), None) == INVALID
    assert b"share" in L.spider_last_error()
