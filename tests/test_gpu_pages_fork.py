"""spider_pages_fork against the oracle: tables, lengths, references and moved slots are equal, bit for bit."""
import numpy as np
import pytest
import torch

from gpu_common import need_gpu
from oracle import paged as op
from paged_common import ints, pages

pytestmark = pytest.mark.gpu


def shared_batch(rng, B, P, M, n_pages, share=0.6, holders=True):
    """Sequences some of whose first pages are another one's; ref counts them and, for some pages, others."""
    lens = rng.integers(0, M * P + 1, B)
    table, ref = np.full((B, M), -1, np.int32), np.zeros(n_pages, np.int64)
    ids = iter(rng.permutation(n_pages))
    for b in range(B):
        pages_b, u = -(-lens[b] // P), rng.integers(0, b) if b else 0
        same = rng.integers(0, min(pages_b, -(-lens[u] // P)) + 1) if b and rng.random() < share else 0
        if same == pages_b and same:
            lens[b] = min(lens[b], lens[u])
            pages_b = -(-lens[b] // P)
            same = min(same, pages_b)
        for i in range(pages_b):
            page = table[u, i] if i < same else next(ids, -1)
            table[b, i] = page
            if page >= 0:
                ref[page] += 1
    if holders:
        held = rng.random(n_pages) < 0.1
        ref[held] += 1
    return table, lens.astype(np.int32), ref.astype(np.int32)


def run(seed, B_in, parent, n_new, P=16, M=6, n_pages=200, L=2, Hkv=2, dh=32, dtype="bf16", heads_first=False, table=None, lens=None, ref=None):
    lib = need_gpu()
    rng = np.random.default_rng(seed)
    if table is None:
        table, lens, ref = shared_batch(rng, B_in, P, M, n_pages)
    k, v = (pages(rng, n_pages, P, Hkv, dh, dtype, heads_first, L) for _ in range(2))
    want = op.pages_fork(table, lens, ref, parent, n_new, P)
    wk, wv = k.clone(), v.clone()
    for src, dst, n in want[4]:
        for x, y in ((wk, k), (wv, v)):
            x[:, dst, :n] = y[:, src, :n]
    t, n, r, m = lib.pages_fork(k, v, ints(table), ints(lens), ints(ref), ints(parent), n_new=None if n_new is None else ints(n_new))
    assert np.array_equal(t.cpu().numpy(), want[0])
    assert np.array_equal(n.cpu().numpy(), want[1])
    assert np.array_equal(r.cpu().numpy(), want[2])
    assert m.item() == want[3]
    assert torch.equal(k, wk) and torch.equal(v, wv)
    return want


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("new", [None, 1, "some"])
def test_random_batches(seed, new):
    rng = np.random.default_rng(100 + seed)
    B_in, B_out = rng.integers(1, 20, 2)
    parent = rng.integers(-2, B_in + 1, B_out)
    n_new = None if new is None else (np.ones(B_out, int) if new == 1 else rng.integers(-3, 40, B_out))
    run(seed, B_in, parent, n_new)


def test_one_prompt_and_four_beams():
    """The first step of a search: the last page has one holder that ends and four that write; the first keeps it."""
    table = np.array([[5, 9, 2, -1]], np.int32)
    ref = np.zeros(12, np.int32)
    ref[[5, 9, 2]] = 1
    want = run(0, 1, [0, 0, 0, 0], [1, 1, 1, 1], M=4, n_pages=12, table=table, lens=np.array([40]), ref=ref)
    assert want[0][:, 2].tolist() == [2, 0, 1, 3] and want[2][2] == 1 and want[2][5] == 4
    assert [c[0] for c in want[4]] == [2, 2, 2]


@pytest.mark.parametrize("outside", [0, 1])
def test_writers_among_other_holders(outside):
    """A page that a sequence without new slots, or somebody outside the batch, holds too is kept by no writer."""
    table = np.array([[3, 4], [3, 4], [3, 4]], np.int32)
    ref = np.array([0, 0, 0, 3, 3 + outside, 0, 0, 0], np.int32)
    run(1, 3, [0, 1, 2], [1, 0, 2], M=2, n_pages=8, table=table, lens=np.array([20, 20, 20]), ref=ref)


def test_full_pages_are_shared_and_not_copied():
    table = np.array([[3, 4, -1]], np.int32)
    ref = np.array([0, 0, 0, 1, 1, 0], np.int32)
    want = run(2, 1, [0, 0], [1, 17], M=3, n_pages=6, table=table, lens=np.array([32]), ref=ref)
    assert not want[4] and want[0].tolist() == [[3, 4, 0], [3, 4, 1]] and want[1].tolist() == [33, 48]


def test_pool_runs_out():
    table = np.array([[0, 1, -1, -1]], np.int32)
    ref = np.array([1, 1, 0], np.int32)
    want = run(3, 1, [0, 0, 0], [20, 1, 40], M=4, n_pages=3, table=table, lens=np.array([20]), ref=ref)
    assert want[3] > 0 and (want[0] == -1).any()


def test_absent_pages_empty_sequences_and_lengths_out_of_range():
    table = np.array([[0, -1, 2], [7, 1 << 30, -(1 << 31)], [3, 4, 5]], np.int32)
    ref = np.array([1, 0, 1, 1, 1, 1, 0, 1, 0], np.int32)
    for lens in ([40, 40, 40], [0, 1 << 30, -4], [33, 17, 48]):
        run(4, 3, [0, 1, 2, 0, 5, -1], [1, 1, 1, 3, 9, 9], M=3, n_pages=9, table=table, lens=np.array(lens), ref=ref)


@pytest.mark.parametrize("B,n_pages,M", [(1, 1, 1), (40, 16384, 300), (40, 16385, 300), (256, 3000, 64), (256, 3000, 65), (300, 5000, 30), (1500, 70000, 40), (4096, 9000, 3)])
def test_large_batches_and_pools(B, n_pages, M):
    rng = np.random.default_rng(B)
    run(B, B, rng.integers(-1, B, B), rng.integers(0, 3, B), P=8, M=M, n_pages=n_pages, L=1, Hkv=1, dh=8)


def test_room_for_long_prompts():
    """Thousands of pages for few sequences, none for others."""
    run(9, 5, [0, 4, -1, 2, 2, 1], [20000, 0, 5000, 9000, 0, 1], P=8, M=4000, n_pages=9000, L=1, Hkv=1, dh=8, table=np.full((5, 4000), -1, np.int32),
        lens=np.zeros(5, int), ref=np.zeros(9000, np.int32))


@pytest.mark.parametrize("P,L,Hkv,dh,dtype,heads_first", [
    (8, 1, 1, 8, "bf16", False), (32, 3, 4, 80, "bf16", True), (64, 2, 3, 4, "f32", False), (256, 2, 2, 256, "f32", True), (4096, 1, 2, 16, "bf16", False),
])
def test_layouts(P, L, Hkv, dh, dtype, heads_first):
    rng = np.random.default_rng(P)
    run(P, 6, rng.integers(0, 6, 9), rng.integers(0, 5, 9), P=P, M=3, n_pages=40, L=L, Hkv=Hkv, dh=dh, dtype=dtype, heads_first=heads_first)


def test_steps_that_follow_each_other_captured():
    """A graph of two forks, from one set of buffers to the other and back, replayed."""
    lib = need_gpu()
    rng = np.random.default_rng(7)
    P, M, n_pages, B = 8, 12, 64, 4
    k, v = (pages(rng, n_pages, P, 2, 32, "f32", False, 2) for _ in range(2))
    table, lens, ref = np.full((B, M), -1, np.int32), np.zeros(B, np.int32), np.zeros(n_pages, np.int32)
    for b in range(B):
        table[b, :3] = [3 * b, 3 * b + 1, 3 * b + 2]
        ref[table[b, :3]] = 1
        lens[b] = 18 + b
    bufs = [[ints(table), ints(lens), ints(ref)], [torch.empty(B, M, dtype=torch.int32).cuda(), torch.empty(B, dtype=torch.int32).cuda(), torch.empty(n_pages, dtype=torch.int32).cuda()]]
    parent, n_new = ints([0, 1, 2, 3]), ints([1] * B)
    missing = torch.zeros(1, dtype=torch.int32).cuda()
    ws = torch.empty(lib.lib().spider_pages_fork_workspace_size(B, n_pages), dtype=torch.uint8, device="cuda")

    def step(k, v, a, b):
        lib.pages_fork(k, v, *a, parent, n_new=n_new, table_out=b[0], lens_out=b[1], ref_out=b[2], missing=missing, workspace=ws)

    step(k.clone(), v.clone(), *bufs)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(k, v, bufs[0], bufs[1])
        step(k, v, bufs[1], bufs[0])
    state, wk, wv = (table, lens, ref), k.clone(), v.clone()
    for p in ([0, 0, 1, 2], [3, 3, 3, 3], [0, 2, 1, -1], [0, 1, 2, 3], [1, 1, 0, 0]):
        parent.copy_(ints(p))
        for _ in range(2):
            *state, _, copies = op.pages_fork(*state, p, [1] * B, P)
            for src, dst, n in copies:
                for x in (wk, wv):
                    x[:, dst, :n] = x[:, src, :n].clone()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(bufs[0], state):
            assert np.array_equal(x.cpu().numpy(), y)
        assert torch.equal(k, wk) and torch.equal(v, wv) and missing.item() == 0
