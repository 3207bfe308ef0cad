"""spider_beam_select against the oracle in 64 bits: beams, tokens, ends and histories are equal; a score is its own
rounding to fp32 off (half a step), and the logarithm of the sum by the exponentials' 2^-23."""
import numpy as np
import pytest
import torch

from gpu_common import need_gpu
from oracle import paged as op
from paged_common import DT, ints

pytestmark = pytest.mark.gpu


def check(x, scores, M, done=None, eos=-1, history=None, n_history=None, seed=0):
    lib = need_gpu()
    kw = {}
    if history is not None:
        out0 = np.random.default_rng(seed).integers(-9, 0, (x.shape[0] * M, history.shape[1])).astype(np.int32)
        kw = dict(history=ints(history), n_history=ints(n_history), history_out=ints(out0))
    got = lib.beam_select(x, torch.from_numpy(np.asarray(scores, np.float32)).cuda(), M, done=None if done is None else ints(done), eos=eos, **kw)
    want = op.beam_select(x.cpu().double().numpy(), np.asarray(scores, np.float32), M, done, eos, history, n_history, out0 if history is not None else None)
    for name in ("parent", "token", "done") + (("history", "n_history") if history is not None else ()):
        assert np.array_equal(got[name].cpu().numpy(), want[name]), name
    g, w = got["scores"].cpu().double().numpy(), want["scores"]
    assert np.array_equal(np.isinf(g), np.isinf(w))
    ok = np.isfinite(w)
    assert (np.abs(g[ok] - w[ok]) <= 2.0 ** -24 * np.abs(w[ok]) + 2.0 ** -23).all()
    return got


def logits(rng, B, K, V, dtype="f32", scale=2.5):
    return torch.from_numpy((scale * rng.standard_normal((B, K, V))).astype(np.float32)).to(DT[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,M,V", [
    (1, 1, 4, 32000), (1, 4, 4, 32000), (3, 5, 5, 32001), (2, 8, 16, 8192), (4, 3, 3, 8193), (2, 2, 64, 500), (1, 64, 64, 20000),
    (2, 17, 33, 40003), (1, 1, 1, 1), (2, 3, 2, 7), (70, 2, 2, 1000), (1, 2, 5, 524288), (1, 32, 32, 160000),
])
def test_sizes(dtype, B, K, M, V):
    rng = np.random.default_rng(V + K)
    check(logits(rng, B, K, V, dtype), rng.uniform(-30, 0, (B, K)), M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("levels", [1, 2, 30])
@pytest.mark.parametrize("V", [300, 9001, 32000])
def test_ties_go_to_the_lower_beam_and_token(dtype, levels, V):
    """Few different logits (one: every candidate alike, more than a piece ranks at once), beams of equal scores."""
    rng = np.random.default_rng(levels)
    x = torch.from_numpy(rng.integers(0, levels, (2, 1, V)).astype(np.float32)).to(DT[dtype]).repeat(1, 3, 1).cuda()
    check(x, np.full((2, 3), -1.5), 7)
    check(x, np.full((2, 3), -1.5), 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_odd_logits(dtype):
    """Rows that a grammar leaves nothing of, NaN, infinities, zeros of both signs, huge and tiny values."""
    rng = np.random.default_rng(1)
    x = logits(rng, 4, 4, 9000, "f32").cpu()
    x[0, 0] = -np.inf
    x[0, 1] = np.nan
    x[0, 2, 17] = np.inf
    x[0, 3, 3:] = -np.inf
    x[1, :, rng.integers(0, 9000, 4000)] = np.nan
    x[1, :, rng.integers(0, 9000, 4000)] = -np.inf
    x[2, 0] = 0.0
    x[2, 1] = -0.0
    x[2, 2, ::2] = -0.0
    x[2, 2, 1::2] = 0.0
    x[2, 3] *= 1e-30
    x[3, 0] *= 1e4
    x[3, 1] = x[3, 1] * 100 + 1e30
    x[3, 2] = -3e38
    x[3, 3] = x[3, 3] - 5e4
    check(x.to(DT[dtype]).cuda(), np.full((4, 4), -2.0) - np.arange(4), 6)


def test_odd_scores_and_too_few_candidates():
    rng = np.random.default_rng(2)
    x = logits(rng, 5, 3, 5)
    scores = np.array([[-np.inf] * 3, [np.nan, -1, np.inf], [-1, -np.inf, -2], [0, 0, 0], [-1e30, 1e30, 3]])
    check(x, scores, 20)
    check(x, scores, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_finished_beams_and_histories(dtype):
    rng = np.random.default_rng(3)
    B, K, V, cap = 6, 4, 3000, 2100
    x = logits(rng, B, K, V, dtype)
    x[:, :, 11] += 8.0  # the end is often among the best
    done = rng.integers(0, 2, (B, K))
    done[0], done[1] = 1, 0
    scores = rng.uniform(-12, -4, (B, K))
    scores[2, 1] = -np.inf
    history = rng.integers(0, V, (B * K, cap)).astype(np.int32)
    n = rng.integers(0, cap + 1, B * K)
    n[:6] = [0, 1, cap, cap - 1, -3, cap + 9]
    check(x, scores, 4, done, 11, history, n)
    check(x, scores, 9, done, 11, history, n)
    check(x, scores, 3, None, 11, history, n)
    check(x, scores, 5, None, -1, history, n)


@pytest.mark.parametrize("M,cap", [(1, 32768), (1, 32769), (4, 8192), (4, 9001), (64, 700)])
def test_long_histories(M, cap):
    rng = np.random.default_rng(cap)
    B, K, V = 2, 3, 500
    history = rng.integers(0, V, (B * K, cap)).astype(np.int32)
    n = np.array([0, cap - 1, cap, 17, cap // 2, 1])
    check(logits(rng, B, K, V), rng.uniform(-2, 0, (B, K)), M, rng.integers(0, 2, (B, K)), 4, history, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows(dtype):
    """Rows of odd width and start within a wider matrix (read one by one), and rows at a distance."""
    rng = np.random.default_rng(4)
    wide = logits(rng, 6, 1, 4111, dtype).view(6, 4111)
    check(wide[:, 3:4003].unflatten(0, (2, 3)), rng.uniform(-9, 0, (2, 3)), 5)
    wide = logits(rng, 6, 1, 4112, dtype).view(6, 4112)
    check(wide[:, 16:4016].unflatten(0, (2, 3)), rng.uniform(-9, 0, (2, 3)), 5)
    check(wide[:, :100].unsqueeze(0), rng.uniform(-9, 0, (1, 6)), 5)


def test_beams_that_differ_by_less_than_fp32_resolves():
    """Scores near -1000 whose candidates differ by about 1e-6: in fp32 they would be equal and come by number."""
    V = 64
    x = torch.zeros(1, 3, V, dtype=torch.float32)
    x[0, :, 1:] = -40.0
    x[0, 1, 0], x[0, 1, 1] = 0.0, -13.0  # e^-13 = 2.3e-6 of its mass elsewhere: beam 1 comes last
    x[0, 0, 1] = -14.0
    got = check(x.cuda(), np.full((1, 3), -1000.0), 3)
    assert got["parent"].cpu().tolist() == [[2, 0, 1]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,M,V", [(16, 16, 9000), (64, 64, 300), (40, 7, 17000), (4, 64, 8200), (64, 4, 5000)])
def test_many_beams(dtype, K, M, V):
    """The bounds of what a beam lists: beams that lead by far, beams alike, finished ones, ones that a grammar leaves
    one token or none, fewer candidates than new beams."""
    rng = np.random.default_rng(K + M)
    x = logits(rng, 6, K, V, dtype).cpu()
    scores = rng.uniform(-4, 0, (6, K))
    scores[0, K // 2] += 40.0  # every new beam from one
    scores[1] = -3.0
    x[1] = x[1, :1]  # ties between beams
    x[2, :, 1:] = -np.inf  # one candidate a beam
    x[3] = -np.inf
    x[3, :2, 5:8] = 1.0  # six
    x[4, ::2] = np.nan
    scores[4, 1::4] = -np.inf
    x[5] = torch.from_numpy(rng.integers(0, 3, (K, V)).astype(np.float32))
    scores[5] = np.round(scores[5])
    done = rng.integers(0, 2, (6, K))
    check(x.cuda(), scores, M)
    check(x.cuda(), scores, M, done, 2)
    check(x.cuda(), scores, M, np.ones((6, K)), 2)


def test_the_largest():
    rng = np.random.default_rng(6)
    check(logits(rng, 1, 64, 524288), rng.uniform(-4, 0, (1, 64)), 64)


def test_same_bits_on_every_call_and_captured():
    lib = need_gpu()
    rng = np.random.default_rng(5)
    B, K, V, cap = 3, 4, 20000, 64
    x, scores = logits(rng, B, K, V), torch.from_numpy(rng.uniform(-9, 0, (B, K)).astype(np.float32)).cuda()
    done, n = ints(np.zeros((B, K))), ints(rng.integers(1, 50, B * K))
    h, ho = ints(rng.integers(0, V, (B * K, cap))), ints(np.zeros((B * K, cap)))
    ws = torch.full((lib.lib().spider_beam_select_workspace_size(B, K, K, V),), 255, dtype=torch.uint8, device="cuda")
    call = lambda out: lib.beam_select(x, scores, K, done=done, eos=2, history=h, n_history=n, history_out=out, workspace=ws)
    call(ho)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call(ho)
    for i in range(4):
        x.copy_(logits(rng, B, K, V))
        done.copy_(ints(rng.integers(0, 2, (B, K))))
        g.replay()
        torch.cuda.synchronize()
        want = call(ho.clone())
        for name in got:
            assert torch.equal(got[name], want[name]), name
