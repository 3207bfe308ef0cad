"""spider_decode_tree: what is refused before anything runs."""
import pytest
import torch

from synth.online_inputs import unembed
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
