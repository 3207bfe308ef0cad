"""spider_decode_tree: many rows against the oracle, and what is refused before anything runs."""
import numpy as np
import pytest
import torch

from oracle import decode as odec
from oracle import drafting as od
from synth.decoder_inputs import layer_weights
from synth.online_inputs import unembed
from gpu_common import log, rel_err
from test_gpu_decode_tree import rows, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wl", ["tiny", "llava15_7b"])
def test_heads_norms_and_caches_of_another_kind_are_refused(wl):
    """The library takes pointers: a head of another type or width would be read past its end."""
    L, dec, bf16, cfg, W, kv = setup(wl, 1, 2, 20)
    x = rows(dec, (2, 3), 1).cuda()
    wu, fn = unembed(dec, 128, seed=3).cuda(), torch.ones(dec.d).cuda()
    other = torch.float32 if bf16 else torch.bfloat16
    L.decode_tree(cfg, W, [5, 0], x, kv, final_norm=fn, w_unembed=wu)
    bad = [dict(w_unembed=wu.to(other)), dict(w_unembed=wu[:, :64].contiguous()), dict(w_unembed=wu.t()), dict(w_unembed=wu.cpu()),
           dict(final_norm=fn.bfloat16()), dict(final_norm=fn[:64].contiguous()), dict(final_norm=fn.cpu()),
           dict(kv={**kv, "k": kv["k"].to(other)}), dict(kv={**kv, "v": kv["v"][:, :1]}), dict(kv={**kv, "v": kv["v"].cpu()})]
    before = kv["k"].clone()
    for kw in bad:
        with pytest.raises(ValueError):
            L.decode_tree(cfg, W, [5, 0], x, **{**dict(kv=kv, final_norm=fn, w_unembed=wu), **kw})
    assert torch.equal(kv["k"], before)


def test_capture_is_refused():
    """Its tables come from a host buffer that the next call fills anew: a replay would read that call's."""
    L, dec, _, cfg, W, kv = setup("tiny", 1, 1, 20)
    x = rows(dec, (1, 3), 2).cuda()
    want, _, _ = L.decode_tree(cfg, W, [5], x, kv)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    table = L.layer_weights(W)
    y = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y.add_(1)
        with pytest.raises(L.SpiderError) as e:
            L.decode_tree(cfg, W, [5], x, kv, weight_table=table, workspace=ws)
    assert "captur" in str(e.value)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert (y == 2).all()
    again, _, _ = L.decode_tree(cfg, W, [5], x, kv)
    assert torch.equal(again, want)


@pytest.mark.parametrize("wl,B,T,lens,evicted", [
    ("llava15_7b", 1, 17, [40], 0), ("llava15_7b", 1, 64, [100], 30), ("llava15_7b", 4, 64, [20, 0, 64, 33], 5),
    ("llava15_7b", 2, 130, [70, 3], 0), ("llava15_7b", 8, 61, [5 * b for b in range(8)], 100), ("tiny", 3, 100, [50, 0, 29], 7),
    ("tiny", 2, 256, [9, 64], 0)])
def test_many_rows_match_the_oracle(wl, B, T, lens, evicted):
    """Rows past 4, 16, 64 and 256, where the products take other kernels, trees of two to four mask words, and
    positions ahead of the slots; bars as in test_gpu_decode_tree.py."""
    cap, V = max(lens) + T + 6, 512
    L, dec, bf16, cfg, W, kv = setup(wl, 1, B, cap)
    rng = np.random.default_rng(T)
    parents = np.stack([[rng.integers(max(-1, t - 9), t) for t in range(T)] for _ in range(B)])
    parents[-1, T - 3:] = -2
    for i, c in enumerate((kv["k"], kv["v"])):
        c.copy_(torch.randn(c.shape, generator=torch.Generator().manual_seed(7 + i)))
    k0, v0 = (c.double().cpu().numpy() for c in (kv["k"], kv["v"]))
    x = rows(dec, (B, T), 3)
    wu, fn = unembed(dec, V, seed=3), torch.rand(dec.d, generator=torch.Generator().manual_seed(5)) + 0.5
    aw = torch.rand(1, B, dec.H, cap).cuda()
    aw0 = aw.double().cpu().numpy()
    pos = [n + evicted for n in lens]
    h, logits, _ = L.decode_tree(cfg, W, lens, x.cuda(), kv, parents=parents, pos=pos, final_norm=fn.cuda(), w_unembed=wu.cuda(),
                                 attn_weights=aw)
    wts = lambda l: {k: v.double().numpy() for k, v in layer_weights(dec, l, 0, "cpu").items()}  # noqa: E731
    recipe = "bf16" if bf16 else "f32"
    ho = od.decode_tree(x.double().numpy(), wts, k0, v0, lens, pos, parents, dec, recipe, aw0)
    lo = odec.lm_head(ho.reshape(B * T, -1), fn.numpy(), wu.double().numpy(), dec.eps, recipe).reshape(B, T, V)
    live = parents > -2
    tol, tol_kv = (2e-2, 1e-2) if bf16 else (1e-4, 1e-5)
    errs = [rel_err(h.cpu().numpy()[live], ho[live]), rel_err(logits.cpu().numpy()[live], lo[live]),
            rel_err(kv["k"].double().cpu().numpy(), k0), rel_err(kv["v"].double().cpu().numpy(), v0), rel_err(aw.double().cpu().numpy(), aw0)]
    log(f"[tree] {wl} {B}x{T}: h, logits, k, v, weights {errs}")
    assert max(errs[0], errs[1], errs[4]) <= tol and max(errs[2], errs[3]) <= tol_kv
