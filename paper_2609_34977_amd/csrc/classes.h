// Kernel classes of the profiler, one bit each in its mask (their names are in host.cpp).  A
// header of its own: the records of profiled traffic name the sources of the kernels they were
// taken on, and a new class changes none of those.
#pragma once

namespace spider {

enum KernelClass {
  KC_SCORE_PREP = 0,
  KC_ANCHOR_TOPK,
  KC_KMEANS,
  KC_MAXSIM,
  KC_SCORE_FINAL,
  KC_SELECT,
  KC_ASSEMBLE,
  KC_EMBED,
  KC_RMSNORM,
  KC_GEMM_QKV,
  KC_QKV_FINALIZE,
  KC_ATTENTION,
  KC_GEMM_O,
  KC_GEMM_GATEUP,
  KC_GEMM_DOWN,
  KC_RESIDUAL,
  KC_LENS_PREP,
  KC_GEMM_LENS,
  KC_LENS_ADMIT,
  KC_COLMEAN,
  KC_CLS_ATTN,
  KC_PROJECTOR,
  KC_LM_HEAD,
  KC_TREE_ATTN,
  KC_TREE_WEIGHTS,
  KC_CACHE_SELECT,
  KC_CACHE_COMPACT,
  KC_ADJUST_LOGITS,
  KC_ROPE_APPEND,
  KC_PAGED_ATTN,
  KC_PAGES_FORK,
  KC_BEAM_SELECT,
  KC_COUNT
};

static_assert(KC_COUNT <= 32, "the profiler's mask has 32 bits");

}  // namespace spider
