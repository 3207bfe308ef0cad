"""spider_rope_append against the oracle in 64 bits.

Tolerance: cosine, sine, one product and the sum are each rounded to fp32 by half a step of values no larger than
|x| + |y| of the pair, four roundings in all, and the result once to its type.
"""
import numpy as np
import pytest
import torch

from gpu_common import need_gpu
from oracle import paged as op
from paged_common import HALF_STEP, batch, f64, ints, pages, rows

pytestmark = pytest.mark.gpu


def pair_sum(x, half):
    s = np.zeros(x.shape)
    s[..., :half] = s[..., half:2 * half] = np.abs(x[..., :half]) + np.abs(x[..., half:2 * half])
    return s


def close(got, want, x, half, dtype):
    tol = HALF_STEP[dtype] * np.abs(want) + 4 * 2.0 ** -24 * pair_sum(x, half)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) - tol)
    assert np.array_equal(got[..., 2 * half:], x[..., 2 * half:])


def tables(rot, sections, inter, theta=10000.0):
    freq, axis = op.rope_axes(rot, theta, sections, inter)
    return freq, axis, torch.from_numpy(freq).cuda(), torch.from_numpy(axis).cuda()


def run(dtype, H, Hkv, dh, rot, sections, inter, lens, news, P, heads_first=False, packed=False, at=0, seed=0, extra_rows=0, shift=0, holes=()):
    lib = need_gpu()
    rng = np.random.default_rng(seed)
    n_pages, table, cu = batch(rng, lens, news, P)
    for b, i in holes:
        table[b, i] = (-1, 1 << 30)[i % 2]
    cu = cu + shift
    N = sum(news) + extra_rows
    kp, vp = (pages(rng, n_pages, P, Hkv, dh, dtype, heads_first) for _ in range(2))
    q, k, v = rows(rng, N, H, dh, dtype, packed=packed), rows(rng, N, Hkv, dh, dtype, packed=packed), rows(rng, N, Hkv, dh, dtype)
    pos = rng.integers(-50, 1000, (len(sections), N)).astype(np.int32) + at
    freq, axis, df, da = tables(rot, sections, inter)
    want = op.rope_append(pos, freq, axis, f64(q), f64(k), f64(v), f64(kp), f64(vp), table, lens, cu)
    q_out = torch.full_like(q, 7.0)
    before = f64(kp), f64(vp)
    lib.rope_append(ints(pos), df, da, q=q, q_out=q_out, k=k, v=v, k_pages=kp, v_pages=vp, table=ints(table), lens=ints(lens), cu_q=ints(cu))
    half, mine = rot // 2, ~np.isnan(want[0])
    close(f64(q_out)[mine].reshape(-1, dh), want[0][mine].reshape(-1, dh), f64(q)[mine].reshape(-1, dh), half, dtype)
    assert (f64(q_out)[~mine] == 7.0).all()
    written = want[2] != before[1]
    slots = written.any((2, 3))
    # a key's bound needs what it was turned from; a slot that nothing went to is as it was
    source = before[0].copy()
    for r, b, p in op.rows_of(lens, cu, N, table.shape[1] * P):
        page = op.page_of(table, b, p // P, n_pages) if p >= 0 else -1
        if page >= 0:
            source[page, p % P] = f64(k)[r]
    close(f64(kp)[slots].reshape(-1, dh), want[1][slots].reshape(-1, dh), source[slots].reshape(-1, dh), half, dtype)
    assert np.array_equal(f64(kp)[~slots], before[0][~slots])
    assert np.array_equal(f64(vp), want[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,dh,rot,sections", [
    (32, 8, 128, 128, [24, 20, 20]), (4, 4, 128, 64, [32]), (6, 2, 48, 40, [8, 6, 6]), (3, 1, 80, 80, [10, 10, 10, 10]),
    (2, 2, 256, 256, [64, 32, 32]), (5, 5, 8, 8, [4]), (2, 1, 16, 2, [1]), (2, 2, 64, 6, [1, 1, 1]), (2, 2, 24, 24, [6, 6]),
])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("lens,news", [([705], [1]), ([70, 9, 100, 3], [70, 1, 33, 2])])
def test_heads_and_axes(dtype, H, Hkv, dh, rot, sections, inter, lens, news):
    run(dtype, H, Hkv, dh, rot, sections, inter, lens, news, 16, seed=dh + rot)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,heads_first,packed,at", [(8, False, True, 0), (64, True, False, 1000000), (256, True, True, 50000), (4096, False, False, 2000000)])
def test_layouts_and_far_positions(dtype, P, heads_first, packed, at):
    run(dtype, 4, 2, 64, 64, [12, 10, 10], True, [300, 8, 77], [290, 8, 5], P, heads_first, packed, at)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1027, 2047, 2048, 2049, 2051])
def test_several_tokens_per_block(dtype, N):
    run(dtype, 2, 1, 32, 32, [6, 5, 5], False, [N - 7, 9], [N - 7, 7], 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_slot(dtype):
    """Absent pages, rows before the first slot, rows of no sequence."""
    run(dtype, 4, 2, 64, 64, [32], False, [64, 40, 5], [50, 40, 9], 16, extra_rows=12, shift=5, holes=[(0, 1), (0, 3), (1, 0)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_alone_in_place_and_keys_alone(dtype):
    lib = need_gpu()
    rng = np.random.default_rng(2)
    freq, axis, df, da = tables(64, [12, 10, 10], True)
    x = rows(rng, 37, 3, 80, dtype)
    pos = rng.integers(0, 500, (3, 37)).astype(np.int32)
    want = np.stack([op.turn(f64(x)[r], pos[:, r], freq, axis) for r in range(37)])
    src = f64(x)
    new = lib.rope_append(ints(pos), df, da, q=x)
    close(f64(new), want, src, 32, dtype)
    assert lib.rope_append(ints(pos), df, da, q=x, q_out=x) is x
    assert torch.equal(x, new)
    n_pages, table, cu = batch(rng, [37], [37], 8)
    kp, vp = (pages(rng, n_pages, 8, 3, 80, dtype) for _ in range(2))
    k = rows(rng, 37, 3, 80, dtype)
    assert lib.rope_append(ints(pos), df, da, k=k, v=x, k_pages=kp, v_pages=vp, table=ints(table), lens=ints([37]), cu_q=ints(cu)) is None
    at = table[0][np.arange(37) // 8], np.arange(37) % 8
    close(f64(kp)[at], np.stack([op.turn(f64(k)[r], pos[:, r], freq, axis) for r in range(37)]), f64(k), 32, dtype)
    assert np.array_equal(f64(vp)[at], f64(x))


def test_one_axis_is_the_decoders_rotation():
    """With one axis and heads of 128 the queries are those of the oracle's decoder."""
    lib = need_gpu()
    from oracle.decoder import rope
    rng = np.random.default_rng(3)
    _, _, df, da = tables(128, [64], False)
    x = rows(rng, 50, 2, 128, "f32")
    want = rope(f64(x), np.arange(50), 10000.0)
    close(f64(lib.rope_append(ints(np.arange(50)[None]), df, da, q=x)), want, f64(x), 64, "f32")


def test_axes_past_the_last_count_as_the_last():
    lib = need_gpu()
    rng = np.random.default_rng(4)
    freq, axis, df, da = tables(32, [8, 8], False)
    da.fill_(200)
    x = rows(rng, 5, 1, 32, "f32")
    pos = rng.integers(0, 500, (2, 5)).astype(np.int32)
    want = np.stack([op.turn(f64(x)[r], pos[:, r], freq, np.full(16, 200)) for r in range(5)])
    close(f64(lib.rope_append(ints(pos), df, da, q=x)), want, f64(x), 16, "f32")


def test_captured():
    lib = need_gpu()
    rng = np.random.default_rng(5)
    freq, axis, df, da = tables(64, [32], False)
    q, k, v = (rows(rng, 6, h, 64, "bf16") for h in (4, 2, 2))
    kp, vp = (pages(rng, 12, 16, 2, 64, "bf16") for _ in range(2))
    pos, t, n, c, qo = ints(np.zeros((1, 6))), ints(np.full((2, 7), -1)), ints([0, 0]), ints([0, 0, 0]), torch.zeros_like(q)
    call = lambda a, b: lib.rope_append(pos, df, da, q=q, q_out=qo, k=k, v=v, k_pages=a, v_pages=b, table=t, lens=n, cu_q=c)
    call(kp.clone(), vp.clone())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(kp, vp)
    for lens, news in (([40, 9], [3, 3]), ([17, 70], [1, 5]), ([6, 0], [6, 0])):
        _, table, cu = batch(rng, lens, news, 16, spare=12 - sum(-(-x // 16) for x in lens))
        t.fill_(-1)
        t[:, :table.shape[1]] = ints(table)
        n.copy_(ints(lens)), c.copy_(ints(cu)), pos.copy_(ints(rng.integers(0, 900, (1, 6))))
        k2, v2 = kp.clone(), vp.clone()
        g.replay()
        torch.cuda.synchronize()
        got = qo.clone()
        call(k2, v2)
        assert torch.equal(kp, k2) and torch.equal(vp, v2) and torch.equal(got, qo)
