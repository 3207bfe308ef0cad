// Rules of a sampler on logits (spider_adjust_logits): penalties for tokens that
// were said before, biases, a grammar mask, and the arg max of what is left.
#include <cmath>

#include "kernels.h"

namespace spider {
namespace {

constexpr int kAdjThreads = 256;
constexpr int kAdjPiece = 4096;          // vocabulary entries per block
constexpr uint32_t kSeen = 0x80000000u;  // count word: the token stands in the prompt

struct AdjustArgs {
  const void* logits;
  float* out;           // or null
  int32_t* next;        // or null
  float2* part;         // [rows][pieces] (largest value, its id as bits)
  const int32_t* history;
  const int32_t* n_history;
  const int32_t* n_prompt;
  const int32_t* n_nodes;
  const int32_t* tokens;  // [B][T] or null
  const uint64_t* tree;
  const float *rep, *freq, *pres;
  const int32_t* bias_ids;
  const float* bias;
  const uint32_t* mask;
  int64_t ls, os, hs, ms;  // row strides: logits, out, history, mask
  int B, T, V, n_bias, pieces;
};

// (value, id) order of the arg max: the larger value, then the lower id.
__device__ __forceinline__ void take_best(float& v, int& i, float v2, int i2) {
  if (v2 > v || (v2 == v && i2 < i)) {
    v = v2;
    i = i2;
  }
}

__device__ __forceinline__ void wave_best(float& v, int& i) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const float v2 = __shfl_xor(v, o, 64);
    const int i2 = __shfl_xor(i, o, 64);
    take_best(v, i, v2, i2);
  }
}

// VEC consecutive logits from p (aligned to VEC of them).
template <typename LT, int VEC>
__device__ __forceinline__ void load_logits(const LT* p, float* x) {
  if constexpr (VEC == 1) {
    if constexpr (sizeof(LT) == 4) x[0] = p[0];
    else x[0] = bf16_bits_to_f32(p[0]);
  } else if constexpr (sizeof(LT) == 4) {
    const floatx4 v = *reinterpret_cast<const floatx4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(v.x << 16);
    x[1] = __uint_as_float(v.x & 0xFFFF0000u);
    x[2] = __uint_as_float(v.y << 16);
    x[3] = __uint_as_float(v.y & 0xFFFF0000u);
  }
}

// One block per (piece of the vocabulary, row): the counts of the piece's tokens in the
// row's history and the places of its biases in LDS, then one pass over the logits, VEC
// at a time (4 where the rows are aligned for it).  Every block reads the whole history
// from L2, which is why the reads go eight at a time.
template <typename LT, int VEC>
__global__ void __launch_bounds__(kAdjThreads) adjust_kernel(AdjustArgs a) {
  __shared__ uint32_t count[kAdjPiece];
  __shared__ int32_t entry[kAdjPiece];  // first bias entry of a token
  __shared__ int twice;                 // some token has several
  __shared__ float bv[kAdjThreads / 64];
  __shared__ int bi[kAdjThreads / 64];
  const int row = blockIdx.y, b = row / a.T, t = row - b * a.T;
  const int tid = threadIdx.x;
  const int nn = a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T;
  if (t >= nn) return;
  const int v0 = blockIdx.x * kAdjPiece, nv = min(kAdjPiece, a.V - v0);
  constexpr int kNone = 0x7fffffff;
  for (int i = tid; i < kAdjPiece / 4; i += kAdjThreads) {
    reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
    if (a.n_bias) reinterpret_cast<int4*>(entry)[i] = make_int4(kNone, kNone, kNone, kNone);
  }
  if (tid == 0) twice = 0;
  __syncthreads();
  if (a.history) {
    const int n = min(max(a.n_history[b], 0), (int)a.hs), np = a.n_prompt ? a.n_prompt[b] : 0;
    const int32_t* h = a.history + b * a.hs;
    for (int i0 = tid; i0 < n; i0 += 8 * kAdjThreads) {
      int32_t id[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) id[u] = h[min(i0 + u * kAdjThreads, n - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + u * kAdjThreads;
        const uint32_t v = (uint32_t)id[u] - (uint32_t)v0;
        if (i < n && v < (uint32_t)nv) {
          if (i < np) atomicOr(&count[v], kSeen);
          else atomicAdd(&count[v], 1u);
        }
      }
    }
  }
  if (a.tokens) {
    const int W = (a.T + 63) / 64;
    const uint64_t* m = a.tree ? a.tree + (int64_t)row * W : nullptr;
    for (int u = tid; u < nn; u += kAdjThreads) {
      const bool sees = m ? (m[u >> 6] >> (u & 63)) & 1 : u <= t;
      const uint32_t v = (uint32_t)a.tokens[(int64_t)b * a.T + u] - (uint32_t)v0;
      if (sees && v < (uint32_t)nv) atomicAdd(&count[v], 1u);
    }
  }
  const int32_t* ids = a.bias_ids + (int64_t)b * a.n_bias;
  const float* bias = a.bias + (int64_t)b * a.n_bias;
  for (int i = tid; i < a.n_bias; i += kAdjThreads) {
    const uint32_t v = (uint32_t)ids[i] - (uint32_t)v0;
    if (v < (uint32_t)nv && atomicMin(&entry[v], i) != kNone) twice = 1;
  }
  const float rep = a.rep ? a.rep[b] : 1.f, freq = a.freq ? a.freq[b] : 0.f, pres = a.pres ? a.pres[b] : 0.f;
  const LT* x = reinterpret_cast<const LT*>(a.logits) + row * a.ls + v0;
  float* o = a.out ? a.out + row * a.os + v0 : nullptr;
  const uint32_t* m = a.mask ? a.mask + row * a.ms + (v0 >> 5) : nullptr;
  float best = -INFINITY;
  int arg = 0x7fffffff;
  __syncthreads();
  const bool again = twice != 0;
  constexpr int UN = VEC == 4 ? 4 : 8;  // loads in flight
  for (int i0 = VEC * tid; i0 < nv; i0 += UN * VEC * kAdjThreads) {
    float z[UN][VEC];
    uint32_t word[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int i = i0 + u * VEC * kAdjThreads;
      if (i < nv) {
        load_logits<LT, VEC>(x + i, z[u]);
        word[u] = m ? m[i >> 5] : ~0u;
      }
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int i = i0 + u * VEC * kAdjThreads;
      if (i >= nv) break;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const uint32_t c = count[i + e];
        float y = z[u][e];
        if (c) y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
        if (c & ~kSeen) y = __fsub_rn(__fsub_rn(y, __fmul_rn(freq, (float)(c & ~kSeen))), pres);
        if (a.n_bias) {
          const int k = entry[i + e];
          float add = 0.f;
          if (k != kNone) {
            add = bias[k];
            if (again)  // the other entries of the token, in order
              for (int j = k + 1; j < a.n_bias; ++j)
                if (ids[j] == v0 + i + e) add = __fadd_rn(add, bias[j]);
          }
          y = __fadd_rn(y, add);
        }
        if (!((word[u] >> ((i + e) & 31)) & 1u)) y = -INFINITY;
        z[u][e] = y;
        if (y > best) {
          best = y;
          arg = v0 + i + e;
        }
      }
      if (o) {
        if constexpr (VEC == 4) *reinterpret_cast<floatx4*>(o + i) = floatx4{z[u][0], z[u][1], z[u][2], z[u][3]};
        else o[i] = z[u][0];
      }
    }
  }
  if (!a.next) return;
  wave_best(best, arg);
  if ((tid & 63) == 0) {
    bv[tid >> 6] = best;
    bi[tid >> 6] = arg;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kAdjThreads / 64; ++w) take_best(best, arg, bv[w], bi[w]);
    a.part[(int64_t)row * a.pieces + blockIdx.x] = make_float2(best, __int_as_float(arg));
  }
}

// A wave per row: the best of its pieces, -1 where nothing is above -inf.
__global__ void __launch_bounds__(64) adjust_join_kernel(AdjustArgs a) {
  const int row = blockIdx.x, b = row / a.T, t = row - b * a.T;
  if (t >= (a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T)) return;
  float best = -INFINITY;
  int arg = 0x7fffffff;
  for (int p = threadIdx.x; p < a.pieces; p += 64) {
    const float2 x = a.part[(int64_t)row * a.pieces + p];
    take_best(best, arg, x.x, __float_as_int(x.y));
  }
  wave_best(best, arg);
  if (threadIdx.x == 0) a.next[row] = best == -INFINITY ? -1 : arg;
}

size_t adjust_ws_bytes(int B, int T, int V) {
  return align_up((size_t)B * T * ceil_div(V, kAdjPiece) * sizeof(float2), 256);
}

bool adjust_shape_ok(int B, int T, int V) {
  return B >= 1 && T >= 1 && T <= 256 && V >= 1 && (int64_t)B * T <= 65535 && V <= (1 << 28);
}

}  // namespace
}  // namespace spider

using namespace spider;

extern "C" size_t spider_adjust_logits_workspace_size(int B, int T, int V) {
  return adjust_shape_ok(B, T, V) ? adjust_ws_bytes(B, T, V) : 0;
}

extern "C" spider_status spider_adjust_logits(
    int B, int T, int V, const void* logits, int64_t logits_stride, spider_dtype dtype, const int32_t* history,
    int64_t history_stride, const int32_t* n_history, const int32_t* n_prompt, const int32_t* n_nodes,
    const int32_t* node_tokens, const uint64_t* tree_mask, const float* repetition, const float* frequency,
    const float* presence, const int32_t* bias_ids, const float* bias, int n_bias, const uint32_t* mask,
    int64_t mask_stride, float* out, int64_t out_stride, int32_t* next_out, void* workspace, size_t workspace_bytes,
    spider_stream stream) {
  clear_error();
  SPIDER_REQUIRE(logits && (out || next_out), SPIDER_ERR_INVALID_ARG,
                 "spider_adjust_logits: logits and out or next_out required");
  SPIDER_REQUIRE(dtype == SPIDER_BF16 || dtype == SPIDER_F32, SPIDER_ERR_INVALID_ARG,
                 "spider_adjust_logits: bad dtype");
  SPIDER_REQUIRE(B >= 1 && T >= 1 && V >= 1 && n_bias >= 0, SPIDER_ERR_INVALID_ARG,
                 "spider_adjust_logits: sizes must be positive");
  SPIDER_REQUIRE(adjust_shape_ok(B, T, V) && n_bias <= 65536, SPIDER_ERR_UNSUPPORTED,
                 "spider_adjust_logits: T <= 256, B * T <= 65535, V <= 2^28, n_bias <= 65536");
  SPIDER_REQUIRE(!history || (n_history && history_stride >= 0 && history_stride <= 0x7fffffff),
                 SPIDER_ERR_INVALID_ARG, "spider_adjust_logits: a history needs n_history and a stride below 2^31");
  SPIDER_REQUIRE(n_bias == 0 || (bias_ids && bias), SPIDER_ERR_INVALID_ARG,
                 "spider_adjust_logits: n_bias without bias_ids and bias");
  SPIDER_REQUIRE(logits_stride >= V && (!out || out_stride >= V), SPIDER_ERR_SHAPE,
                 "spider_adjust_logits: rows of %d values need strides of at least as many", V);
  SPIDER_REQUIRE(!mask || mask_stride == 0 || mask_stride >= (V + 31) / 32, SPIDER_ERR_SHAPE,
                 "spider_adjust_logits: mask_stride must be 0 or hold (V + 31) / 32 words");
  SPIDER_REQUIRE(out != logits || (dtype == SPIDER_F32 && out_stride == logits_stride), SPIDER_ERR_INVALID_ARG,
                 "spider_adjust_logits: in place needs fp32 logits and equal strides");
  const uintptr_t low = dtype == SPIDER_BF16 ? 1 : 3;
  SPIDER_REQUIRE((reinterpret_cast<uintptr_t>(logits) & low) == 0 && reinterpret_cast<uintptr_t>(out) % 4 == 0,
                 SPIDER_ERR_INVALID_ARG, "spider_adjust_logits: logits and out must be aligned to their types");
  const size_t need = next_out ? adjust_ws_bytes(B, T, V) : 0;
  SPIDER_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), SPIDER_ERR_WORKSPACE,
                 "spider_adjust_logits: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : 0);
  SPIDER_REQUIRE(need == 0 || reinterpret_cast<uintptr_t>(workspace) % 256 == 0, SPIDER_ERR_INVALID_ARG,
                 "spider_adjust_logits: workspace must be 256-byte aligned");
  const AdjustArgs a{logits, out, next_out, reinterpret_cast<float2*>(workspace), history, n_history, n_prompt,
                     n_nodes, node_tokens, tree_mask, repetition, frequency, presence, bias_ids, bias, mask,
                     logits_stride, out_stride, history_stride, mask_stride, B, T, V, n_bias, ceil_div(V, kAdjPiece)};
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  ProfScope ps(KC_ADJUST_LOGITS, st);
  const dim3 grid((unsigned)a.pieces, (unsigned)(B * T));
  // four logits at a time where every row starts on a 16-byte (bf16: 8-byte) boundary and has a multiple of 4
  const uintptr_t four = dtype == SPIDER_BF16 ? 7 : 15;
  const bool vec = V % 4 == 0 && logits_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(logits) & four) == 0 &&
                   (!out || (out_stride % 4 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0));
  if (dtype == SPIDER_BF16) {
    if (vec) adjust_kernel<uint16_t, 4><<<grid, kAdjThreads, 0, st>>>(a);
    else adjust_kernel<uint16_t, 1><<<grid, kAdjThreads, 0, st>>>(a);
  } else {
    if (vec) adjust_kernel<float, 4><<<grid, kAdjThreads, 0, st>>>(a);
    else adjust_kernel<float, 1><<<grid, kAdjThreads, 0, st>>>(a);
  }
  SPIDER_LAUNCHED("adjust_logits");
  if (next_out) {
    adjust_join_kernel<<<(unsigned)(B * T), 64, 0, st>>>(a);
    SPIDER_LAUNCHED("adjust_join");
  }
  return SPIDER_OK;
}
