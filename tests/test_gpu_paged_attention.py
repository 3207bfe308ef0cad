"""spider_paged_attention against the oracle in 64 bits.

Tolerance of an output o of a row that sees n slots: its own rounding, half a step of |o|; in bf16 every weight
rounded by half a step with their sum taken of the rounded ones, half a step of sum_j p_j |v_j - o|; and the fp32
parts: a score is off by at most (dh + 4) 2^-24 of sum_c |scale q_c k_c| (dh additions, the scale, the difference to
the maximum), an exponential by 2^-22 more, each of which moves a weight and the sum, and n additions by n 2^-24.
"""
import numpy as np
import pytest
import torch

from gpu_common import need_gpu
from oracle import paged as op
from paged_common import HALF_STEP, batch, f64, ints, pages, rows

pytestmark = pytest.mark.gpu


def check(got, q, kp, vp, table, lens, cu, dtype, window=0, scale=None, left=None):
    want, spread, size, reach = op.paged_attention(f64(q), f64(kp), f64(vp), table, lens, cu, window, scale)
    dh, g = q.shape[2], f64(got)
    nobody = np.isnan(want)
    if left is not None:
        assert np.array_equal(g[nobody], np.broadcast_to(left, g.shape)[nobody])
    else:
        assert not nobody.any()
    fp32 = (2 * ((dh + 4) * 2.0 ** -24 * reach[..., :1] + 2.0 ** -22) + reach[..., 1:] * 2.0 ** -24) * size
    tol = HALF_STEP[dtype] * (np.abs(want) + (spread if dtype == "bf16" else 0.0)) + fp32
    worst = np.nanmax(np.abs(g - want) / np.maximum(tol, 1e-30))
    assert not np.isnan(g[~nobody]).any() and worst <= 1.0, worst
    return worst


def case(seed, H, Hkv, dh, P, lens, news, dtype, heads_first=False, packed=False, q_scale=1.5, extra_rows=0):
    rng = np.random.default_rng(seed)
    n_pages, table, cu = batch(rng, lens, news, P)
    kp, vp = (pages(rng, n_pages, P, Hkv, dh, dtype, heads_first) for _ in range(2))
    q = rows(rng, sum(news) + extra_rows, H, dh, dtype, q_scale, packed)
    return q, kp, vp, table, cu


HEADS = [(4, 4, 128), (8, 2, 128), (6, 2, 48), (4, 1, 256), (3, 3, 80), (2, 2, 64), (5, 1, 16), (2, 2, 8), (2, 1, 136)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,dh", HEADS)
@pytest.mark.parametrize("lens,news", [
    ([1], [1]),
    ([200, 33, 1, 64], [1, 1, 1, 1]),
    ([70, 8, 100], [70, 3, 17]),
    ([31, 0, 65], [5, 0, 40]),
    ([300], [130]),
    ([90] * 70, [1] * 70),
])
def test_head_layouts(dtype, H, Hkv, dh, lens, news):
    lib = need_gpu()
    q, kp, vp, table, cu = case(dh + len(lens), H, Hkv, dh, 16, lens, news, dtype)
    out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu))
    check(out, q, kp, vp, table, lens, cu, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [8, 16, 32, 64, 256, 4096])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("window", [0, 1, 37, 300])
def test_page_sizes_layouts_and_windows(dtype, P, heads_first, window):
    lib = need_gpu()
    lens, news = [530, 17, 256], [60, 17, 1]
    q, kp, vp, table, cu = case(P + window, 4, 2, 64, P, lens, news, dtype, heads_first, packed=True)
    out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), window=window)
    check(out, q, kp, vp, table, lens, cu, dtype, window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257])
@pytest.mark.parametrize("dh", [64, 128, 256])
def test_chunk_sizes(dtype, T, dh):
    """Both sides of every row count that another kernel or tile takes over at."""
    lib = need_gpu()
    lens, news = [T + 45, T], [T, max(1, T - 1)]
    q, kp, vp, table, cu = case(T, 2, 1, dh, 32, lens, news, dtype)
    out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu))
    check(out, q, kp, vp, table, lens, cu, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,news,H,Hkv,dh", [
    ([4000], [1], 4, 2, 128),
    ([4000, 300, 9, 2047], [1, 1, 1, 1], 8, 8, 128),
    ([3000], [40], 2, 1, 64),
    ([2999, 5], [100, 5], 2, 1, 128),
    ([5000], [2], 3, 1, 256),
])
def test_splits(dtype, lens, news, H, Hkv, dh):
    lib = need_gpu()
    q, kp, vp, table, cu = case(len(lens), H, Hkv, dh, 16, lens, news, dtype)
    need = lib.lib().spider_paged_attention_workspace_size(sum(news), len(lens), H, Hkv, dh, table.shape[1] * 16, lib.BF16 if dtype == "bf16" else lib.F32)
    assert need > 0  # the keys are split
    for window in (0, 777):
        out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), window=window)
        check(out, q, kp, vp, table, lens, cu, dtype, window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_uneven_batches(dtype):
    """A batch whose average says nothing: one long chunk among single tokens, all rows in one sequence, none in others."""
    lib = need_gpu()
    for lens, news in (([600] + [70] * 9, [150] + [1] * 9), ([70] * 9 + [600], [0] * 9 + [9]), ([5] * 30 + [200], [0] * 30 + [100]),
                       ([100] * 100, [0, 1] * 50)):
        q, kp, vp, table, cu = case(len(lens), 4, 2, 128, 16, lens, news, dtype)
        out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu))
        check(out, q, kp, vp, table, lens, cu, dtype)


@pytest.mark.parametrize("B", [63, 64, 65, 4096, 4100])
def test_many_sequences(B):
    """The search for a row's sequence goes over one, two and three rounds."""
    lib = need_gpu()
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 20, B)
    news = np.minimum(rng.integers(0, 4, B), lens)
    q, kp, vp, table, cu = case(B, 2, 1, 64, 8, lens.tolist(), news.tolist(), "bf16")
    out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu))
    check(out, q, kp, vp, table, lens, cu, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1], [70, 40, 3]])
def test_absent_pages_and_rows_that_see_nothing(dtype, news):
    lib = need_gpu()
    lens = [160, 41, 2]
    q, kp, vp, table, cu = case(5, 4, 2, 64, 16, lens, news, dtype)
    table[0, [0, 3, 4]] = -1
    table[0, 9] = 1 << 30      # outside the pool: absent too
    table[1, :] = -(1 << 31)   # no page at all
    lens[2] = 2 - news[2] // 3 - 1  # rows before the first slot
    for window in (0, 16):
        out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), window=window)
        check(out, q, kp, vp, table, lens, cu, dtype, window)
        assert (f64(out)[cu[1]:cu[2]] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [90, 33]])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_what_a_row_does_not_see_does_not_matter(dtype, news, bad):
    """Slots behind the position, before the window, of other sequences and of no sequence hold infinities and NaN."""
    lib = need_gpu()
    lens, P, window = [150, 70], 16, 40
    q, kp, vp, table, cu = case(6, 4, 2, 128, P, lens, news, dtype)
    table[0, 2] = -1
    seen = np.zeros((kp.shape[0], P), bool)
    for b, n in enumerate(lens):
        for j in range(max(0, n - news[b] - window + 1), n):
            if table[b, j // P] >= 0:
                seen[table[b, j // P], j % P] = True
    clean = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), window=window)
    check(clean, q, kp, vp, table, lens, cu, dtype, window)
    hole = torch.from_numpy(~seen).cuda()
    kp[hole] = bad
    vp[hole] = bad
    out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), window=window)
    assert torch.equal(out, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 7, 60, 200])
def test_infinite_and_nan_values_reach_the_rows_that_see_them_and_no_other(dtype, T):
    lib = need_gpu()
    lens, news = [T + 300], [T]
    q, kp, vp, table, cu = case(T, 4, 2, 128, 16, lens, news, dtype)
    base = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu))
    for j, bad in ((lens[0] - 1, np.inf), (lens[0] - max(1, T // 2), np.nan), (lens[0] - T, -np.inf), (3, np.nan)):
        v2 = vp.clone()
        v2[table[0, j // 16], j % 16, 1, 5] = bad
        out = f64(lib.paged_attention(q, kp, v2, ints(table), ints(lens), ints(cu)))
        want = f64(base)
        for r in range(T):
            sees = lens[0] - T + r >= j
            assert np.isfinite(out[r, 2:, 5]).any() != sees
            want[r, 2:, 5] = out[r, 2:, 5]
        assert np.array_equal(out, want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [7, 30, 60, 100, 200])
def test_nan_queries_and_keys_stay_with_their_rows(dtype, T):
    """A NaN in one row's query, and an infinite key that only the last rows see, change no other row."""
    lib = need_gpu()
    lens, news = [T + 100], [T]
    q, kp, vp, table, cu = case(T + 1, 2, 2, 128, 16, lens, news, dtype)
    args = (ints(table), ints(lens), ints(cu))
    base = lib.paged_attention(q, kp, vp, *args)
    for r in (0, T // 2, T - 1):
        q2 = q.clone()
        q2[r, 1, 77] = float("nan")
        out = lib.paged_attention(q2, kp, vp, *args)
        assert torch.isnan(out[r, 1]).all()
        out[r, 1] = base[r, 1]
        assert torch.equal(out, base)
    j = lens[0] - 3
    k2 = kp.clone()
    k2[table[0, j // 16], j % 16, 0, 3] = float("nan")
    out = lib.paged_attention(q, k2, vp, *args)
    assert torch.isnan(out[T - 3:, 0]).all()
    out[T - 3:, 0] = base[T - 3:, 0]
    assert torch.equal(out, base)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 40, 90])
def test_the_largest_window(dtype, T):
    lib = need_gpu()
    q, kp, vp, table, cu = case(T, 2, 1, 64, 16, [T + 9], [T], dtype)
    args = (ints(table), ints([T + 9]), ints(cu))
    assert torch.equal(lib.paged_attention(q, kp, vp, *args, window=2**31 - 1), lib.paged_attention(q, kp, vp, *args))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 4.0])
def test_scales(dtype, scale):
    lib = need_gpu()
    lens, news = [100, 40], [33, 1]
    q, kp, vp, table, cu = case(8, 4, 2, 64, 32, lens, news, dtype)
    out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), scale=scale)
    check(out, q, kp, vp, table, lens, cu, dtype, scale=scale)


@pytest.mark.parametrize("dh", [64, 128, 256])
@pytest.mark.parametrize("T", [130, 400, 800])
def test_few_rows_among_chunks(dh, T):
    """Single tokens, some tokens, none and a chunk in one batch, over pages whose free slots hold anything: equal
    bits with NaN and infinities there."""
    lib = need_gpu()
    lens, news = [1000, 33, T + 40, 500, 77, 1, 2100], [1, 4, T, 0, 17, 1, 8]
    q, kp, vp, table, cu = case(dh + T, 4, 2, dh, 16, lens, news, "bf16", packed=True)
    out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu))
    check(out, q, kp, vp, table, lens, cu, "bf16")
    free = np.ones((kp.shape[0], 16), bool)
    for b, n in enumerate(lens):
        for j in range(n):
            free[table[b, j // 16], j % 16] = False
    free = torch.from_numpy(free).cuda()
    for bad in (float("nan"), float("inf")):
        kp[free] = bad
        vp[free] = -bad
        assert torch.equal(lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu)), out)
        window = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), window=90)
        kp[free] = 0.0
        vp[free] = 0.0
        check(window, q, kp, vp, table, lens, cu, "bf16", 90)


@pytest.mark.parametrize("dh", [24, 80, 120, 200])
@pytest.mark.parametrize("T", [40, 100, 200])
def test_chunks_narrower_than_the_kernel(dh, T):
    """One sequence, and one among others of a few tokens (G = 2 rows per token: blocks of 64 to 256 rows)."""
    lib = need_gpu()
    for lens, news in (([T + 150], [T]), ([T + 33, 900, T, 70], [T, 2, T, 8])):
        q, kp, vp, table, cu = case(dh + T, 4, 2, dh, 16, lens, news, "bf16")
        out = lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu))
        check(out, q, kp, vp, table, lens, cu, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, -1.0])
@pytest.mark.parametrize("news", [1, 40, 240])
def test_the_largest_scores(dtype, scale, news):
    """Scores of 2^20 to 2^28, 2^20 apart: every weight but the largest is 0 (e^-2^20), so the output is the value of
    that slot: one product, one division and its own rounding off."""
    lib = need_gpu()
    n, H, dh = 250, 4, 128
    q, kp, vp, table, cu = case(news, H, 2, dh, 16, [n], [news], dtype)
    order = np.random.default_rng(news).permutation(n) + 1.0
    q[:, :, 0] = 2.0 ** 20
    kp.zero_()
    v, first = f64(vp), n - news
    for j in range(n):
        kp[int(table[0, j // 16]), j % 16, :, 0] = float(order[j])
    got = f64(lib.paged_attention(q, kp, vp, ints(table), ints([n]), ints(cu), scale=scale))
    for r in range(news):
        seen = order[:first + r + 1]
        j = int(seen.argmax() if scale > 0 else seen.argmin())
        want = np.repeat(v[int(table[0, j // 16]), j % 16], H // 2, axis=0)
        assert (np.abs(got[r] - want) <= (HALF_STEP[dtype] + 2.0 ** -22) * np.abs(want)).all(), r


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_scores_of_a_long_row(dtype):
    """All weights alike, far more of them than the mantissa of the sum's type has steps."""
    lib = need_gpu()
    n, P = 20000, 64
    rng = np.random.default_rng(3)
    n_pages, table, cu = batch(rng, [n], [1], P)
    kp = torch.zeros(n_pages, P, 1, 64, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    vp = torch.full_like(kp, 1.0)
    q = rows(rng, 1, 1, 64, dtype)
    out = lib.paged_attention(q, kp, vp, ints(table), ints([n]), ints(cu))
    assert torch.equal(out, torch.ones_like(out))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_sequence_are_left(dtype):
    lib = need_gpu()
    lens, news = [50, 60], [4, 30]
    q, kp, vp, table, cu = case(9, 4, 2, 64, 16, lens, news, dtype, extra_rows=11)
    cu = cu + 5
    out = torch.full_like(q, 7.0)
    lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(cu), out=out)
    check(out, q, kp, vp, table, lens, cu, dtype, left=7.0)


def test_lengths_past_the_table_and_broken_boundaries_stay_in_bounds():
    """Arrays that no program should hold: the call reads and writes nothing outside its tensors."""
    lib = need_gpu()
    lens, news = [64, 64], [20, 20]
    q, kp, vp, table, cu = case(10, 4, 2, 64, 16, lens, news, "bf16")
    out = lib.paged_attention(q, kp, vp, ints(table), ints([1 << 30, -5]), ints(cu))
    check(out, q, kp, vp, table, [1 << 30, -5], cu, "bf16")
    for broken in ([0, -7, 40], [-3, 20, 1 << 30], [0, 20, 40]):
        out = torch.full_like(q, 7.0)
        lib.paged_attention(q, kp, vp, ints(table), ints(lens), ints(broken), out=out)
        if broken[1] > 0:
            check(out, q, kp, vp, table, lens, np.clip(broken, 0, 40), "bf16", left=7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_on_every_call_stream_and_workspace(dtype):
    lib = need_gpu()
    lens, news = [3000, 500], [3, 1]
    q, kp, vp, table, cu = case(11, 4, 2, 128, 16, lens, news, dtype)
    t, n, c = ints(table), ints(lens), ints(cu)
    first = lib.paged_attention(q, kp, vp, t, n, c)
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(first, lib.paged_attention(q, kp, vp, t, n, c, workspace=ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = lib.paged_attention(q, kp, vp, t, n, c)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, other)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_calls_follow_the_tables(dtype):
    """Two captured graphs with a workspace each, replayed with other lengths, pages and boundaries."""
    lib = need_gpu()
    P, B, N = 16, 3, 40
    rng = np.random.default_rng(12)
    kp, vp = (pages(rng, 60, P, 2, 64, dtype) for _ in range(2))
    q = rows(rng, N, 4, 64, dtype, 1.5)
    t, n, c = ints(np.full((B, 24), -1)), ints([0] * B), ints([0] * (B + 1))
    size = lib.lib().spider_paged_attention_workspace_size(N, B, 4, 2, 64, 24 * P, lib.BF16 if dtype == "bf16" else lib.F32)
    graphs = []
    for window in (0, 50):
        ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
        out = torch.zeros_like(q)
        lib.paged_attention(q, kp, vp, t, n, c, window=window, out=out, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            lib.paged_attention(q, kp, vp, t, n, c, window=window, out=out, workspace=ws)
        graphs.append((g, out, window, ws))
    for lens, news in (([300, 17, 9], [30, 1, 9]), ([40, 250, 1], [1, 36, 1]), ([13, 0, 310], [13, 0, 2])):
        _, table, cu = batch(rng, lens, news, P, spare=60 - sum(-(-x // P) for x in lens))
        t.fill_(-1)
        t[:, :table.shape[1]] = ints(table)
        n.copy_(ints(lens))
        c.copy_(ints(cu))
        for g, out, window, _ in graphs:
            out.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            check(out, q, kp, vp, t.cpu().numpy(), lens, cu, dtype, window, left=7.0)


def test_pages_past_2_31_elements():
    """Offsets that do not fit 32 bits: the last pages of a cache of 5 GB."""
    lib = need_gpu()
    P, dh, n_pages = 4096, 128, 4800
    kp = torch.zeros(n_pages, P, 1, dh, dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    rng = np.random.default_rng(13)
    for x in (kp, vp):
        x[-1] = torch.from_numpy(rng.standard_normal((P, 1, dh)).astype(np.float32)).cuda()
    for news in ([1], [40], [100]):
        q = rows(rng, news[0], 2, dh, "bf16", 1.5)
        table = np.array([[n_pages - 1, -1]], np.int32)
        out = lib.paged_attention(q, kp, vp, ints(table), ints([150]), ints([0, news[0]]))
        check(out, q, kp[-1:], vp[-1:], np.array([[0, -1]]), [150], [0, news[0]], "bf16")
