"""MI355X (gfx950) implementation of SPIDER's pruned-and-skipped multimodal prefill.

The work happens in libspider.so (hand-written HIP kernels behind the C ABI of
include/spider.h); this package only loads it and marshals torch tensors.
"""
from ._lib import (  # noqa: F401
    BF16, F32, SpiderError, adjust_logits, budget, cache_compact, cache_select, decode_tree, decoder_cfg,
    layer_weights, lib, plan_skips, prefill, prefill_workspace_size, profile_enable, profile_read, score, select,
    slc_policy, tree_attention, tree_mask,
)
from .pipeline import Pipeline  # noqa: F401
