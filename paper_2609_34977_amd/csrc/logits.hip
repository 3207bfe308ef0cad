// Rules of a sampler on logits (spider_adjust_logits): penalties for tokens that
// were said before, biases, a grammar mask, and the arg max of what is left.
// One reading and one writing of the logits.  Measured on one MI355X: 248 rows of 32000
// (fp32, mask, 100 biases, 2900 tokens) 18.0 us, 3.5 TB/s; 64 rows of 151000 (bf16, 300
// biases, 12000 tokens) 25.9 us, 2.3 TB/s; one row of 32000 11.0 us.
#include <cmath>

#include "kernels.h"

namespace spider {
namespace {

constexpr uint32_t kSeen = 0x80000000u;  // count word: the token stands in the prompt
// A row's history: the kernel's index runs up to 8 * 1024 past its end, and the counts of it
// and of 256 nodes stay below kSeen.
constexpr int64_t kMaxHistory = (1ll << 31) - (1 << 14);

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

// A logit under the penalties: c is the count word of its token.
__device__ __forceinline__ float penalised(float y, uint32_t c, float rep, float freq, float pres) {
  if (c) y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
  if (c & ~kSeen) y = __fsub_rn(__fsub_rn(y, __fmul_rn(freq, (float)(c & ~kSeen))), pres);
  return y;
}

// The bias entries of a token, added up in list order by a wave: 64 entries per load, 8 loads
// in flight.  One token named twice in 8 lists of 1500 / 32000, whole call: 13 / 72 us; with
// a lane looking through the list for its token, 16 loads in flight, 77 / 1430.
__device__ __forceinline__ float bias_of(int token, const int32_t* ids, const float* bias, int n) {
  const int lane = threadIdx.x & 63;
  float add = 0.f;
#pragma unroll 1
  for (int j0 = 0; j0 < n; j0 += 8 * 64) {
    int32_t id[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) id[u] = ids[min(j0 + 64 * u + lane, n - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      uint64_t hit = __ballot(j0 + 64 * u + lane < n && id[u] == token);
      for (; hit; hit &= hit - 1) add = __fadd_rn(add, bias[j0 + 64 * u + __ffsll((unsigned long long)hit) - 1]);
    }
  }
  return add;
}

// One block per (piece of the vocabulary, row): the counts of the piece's tokens in the
// row's history in LDS, then one pass over the logits, VEC at a time (4 where the rows are
// aligned for it), all of a thread's on their way while the counts are made; then the few
// tokens with a bias, which that pass leaves out (bits in LDS), each by the thread that
// marked it.  A piece is as large as its counts fit: every block reads the whole history,
// and a row in one piece needs no second launch for its arg max.
template <typename LT, int VEC, int PIECE, int THREADS>
__global__ void __launch_bounds__(THREADS) adjust_kernel(AdjustArgs a) {
  constexpr int UN = PIECE / THREADS / VEC;
  __shared__ uint32_t count[PIECE];
  __shared__ uint32_t biased[PIECE / 32], twice[PIECE / 32];  // tokens with a bias entry, with several
  __shared__ float bv[THREADS / 64];
  __shared__ int bi[THREADS / 64];
  const int row = blockIdx.y, b = row / a.T, t = row - b * a.T;
  const int tid = threadIdx.x;
  const int nn = a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T;
  if (t >= nn) return;
  const int v0 = blockIdx.x * PIECE, nv = min(PIECE, a.V - v0);
  const LT* x = reinterpret_cast<const LT*>(a.logits) + row * a.ls + v0;
  const uint32_t* m = a.mask ? a.mask + row * a.ms + (v0 >> 5) : nullptr;
  float* o = a.out ? a.out + row * a.os + v0 : nullptr;
  float z[UN][VEC];
  uint32_t word[UN];
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    const int i = VEC * (tid + u * THREADS);
    if (i < nv) {
      load_logits<LT, VEC>(x + i, z[u]);
      word[u] = m ? m[i >> 5] : ~0u;
    }
  }
  for (int i = tid; i < min(PIECE, (nv + 3) & ~3) / 4; i += THREADS) reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
  for (int i = tid; i < PIECE / 32; i += THREADS) biased[i] = twice[i] = 0;
  __syncthreads();
  if (a.history) {
    const int n = min(max(a.n_history[b], 0), (int)a.hs), np = a.n_prompt ? a.n_prompt[b] : 0;
    const int32_t* h = a.history + b * a.hs;
    for (int i0 = tid; i0 < n; i0 += 8 * THREADS) {
      int32_t id[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) id[u] = h[min(i0 + u * THREADS, n - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + u * THREADS;
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
    const uint64_t* tr = a.tree ? a.tree + (int64_t)row * W : nullptr;
    for (int u = tid; u < nn; u += THREADS) {
      const bool sees = tr ? (tr[u >> 6] >> (u & 63)) & 1 : u <= t;
      const uint32_t v = (uint32_t)a.tokens[(int64_t)b * a.T + u] - (uint32_t)v0;
      if (sees && v < (uint32_t)nv) atomicAdd(&count[v], 1u);
    }
  }
  const int32_t* ids = a.bias_ids + (int64_t)b * a.n_bias;
  const float* bias = a.bias + (int64_t)b * a.n_bias;
  uint64_t mine = 0;  // which of this thread's first 64 entries marked their token
  for (int i = tid, k = 0; i < a.n_bias; i += THREADS, ++k) {
    const uint32_t v = (uint32_t)ids[i] - (uint32_t)v0;
    if (v >= (uint32_t)nv) continue;
    if (atomicOr(&biased[v >> 5], 1u << (v & 31)) >> (v & 31) & 1u) atomicOr(&twice[v >> 5], 1u << (v & 31));
    else mine |= 1ull << k;
  }
  const float rep = a.rep ? a.rep[b] : 1.f, freq = a.freq ? a.freq[b] : 0.f, pres = a.pres ? a.pres[b] : 0.f;
  float best = -INFINITY;
  int arg = 0x7fffffff;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    const int i = VEC * (tid + u * THREADS);
    if (i >= nv) break;
    const uint32_t skip = a.n_bias ? biased[i >> 5] >> (i & 31) : 0u;
    uint32_t c[VEC], any = 0;  // few tokens of a vocabulary were said: one test for VEC of them
#pragma unroll
    for (int e = 0; e < VEC; ++e) any |= c[e] = count[i + e];
    if (any) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[u][e] = penalised(z[u][e], c[e], rep, freq, pres);
    }
    const uint32_t allowed = word[u] >> (i & 31);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float y = z[u][e];
      if (a.n_bias) y = __fadd_rn(y, 0.f);
      if (!((allowed >> e) & 1u)) y = -INFINITY;
      z[u][e] = y;
      if (y > best && !((skip >> e) & 1u)) {
        best = y;
        arg = v0 + i + e;
      }
    }
    if (o) {
      if (VEC == 4 && (skip & 15u) == 0) {
        *reinterpret_cast<floatx4*>(o + i) = floatx4{z[u][0], z[u][VEC > 1 ? 1 : 0], z[u][VEC > 2 ? 2 : 0], z[u][VEC > 3 ? 3 : 0]};
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (!((skip >> e) & 1u)) o[i + e] = z[u][e];
      }
    }
  }
  for (int i = tid; __any(mine != 0); i += THREADS, mine >>= 1) {
    const bool on = mine & 1u;
    const int v = on ? ids[i] - v0 : 0;
    float add = on ? __fadd_rn(0.f, bias[i]) : 0.f, y[1];
    uint64_t several = __ballot(on && ((twice[v >> 5] >> (v & 31)) & 1u));
    for (; several; several &= several - 1) {  // the wave adds up one lane's token after the other
      const int lane = __ffsll((unsigned long long)several) - 1;
      const float sum = bias_of(__builtin_amdgcn_readlane(v0 + v, lane), ids, bias, a.n_bias);
      if ((tid & 63) == lane) add = sum;
    }
    if (!on) continue;
    load_logits<LT, 1>(x + v, y);
    float w = __fadd_rn(penalised(y[0], count[v], rep, freq, pres), add);
    if (m && !((m[v >> 5] >> (v & 31)) & 1u)) w = -INFINITY;
    if (o) o[v] = w;
    take_best(best, arg, w, w != w || w == -INFINITY ? 0x7fffffff : v0 + v);
  }
  if (!a.next) return;
  wave_best(best, arg);
  if ((tid & 63) == 0) {
    bv[tid >> 6] = best;
    bi[tid >> 6] = arg;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < THREADS / 64; ++w) take_best(best, arg, bv[w], bi[w]);
    if (a.pieces == 1) a.next[row] = best == -INFINITY ? -1 : arg;
    else a.part[(int64_t)row * a.pieces + blockIdx.x] = make_float2(best, __int_as_float(arg));
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

// Pieces of a row: all of it where its counts fit the LDS of a CU (a block per CU, but one
// launch, one reading of the history and no workspace), else 8192 tokens, four blocks per
// CU; and rows of up to 8192 in such blocks too.  Measured, pieces of 8192 / 32768, us.
// Whole calls: 1 row of 32000 14.7 / 11.8 (the host's second launch); 64 rows of 151000 with
// 12000 tokens of history 26.7 / 35.0 (16384: 33.2, in 1024 threads 28.3).  On the device,
// histories of 2900: 1 row of 32000 9.3 / 12.3, 64 rows 11.6 / 15.2, 248 21.6 / 19.6, 300
// 25.7 / 32.0, 1024 64 / 74; 248 rows of 12000 14.8 / 11.4: past the 256 CUs pieces would be
// faster, at the price of a workspace.
constexpr int kPiece = 8192, kRow = 32768, kMaxBias = 64 * 512;
int adjust_piece(int V) { return V > kPiece && V <= kRow ? kRow : kPiece; }

template <typename LT, int VEC>
void launch_adjust(const AdjustArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.pieces, (unsigned)(a.B * a.T));
  if (adjust_piece(a.V) == kRow) adjust_kernel<LT, VEC, kRow, 1024><<<grid, 1024, 0, st>>>(a);
  else adjust_kernel<LT, VEC, kPiece, 512><<<grid, 512, 0, st>>>(a);
}

size_t adjust_ws_bytes(int B, int T, int V) {
  const int pieces = ceil_div(V, adjust_piece(V));
  return pieces == 1 ? 0 : align_up((size_t)B * T * pieces * sizeof(float2), 256);
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
  SPIDER_REQUIRE(adjust_shape_ok(B, T, V) && n_bias <= kMaxBias, SPIDER_ERR_UNSUPPORTED,
                 "spider_adjust_logits: T <= 256, B * T <= 65535, V <= 2^28, n_bias <= 32768");
  SPIDER_REQUIRE(!history || (n_history && history_stride >= 0 && history_stride <= kMaxHistory),
                 SPIDER_ERR_INVALID_ARG,
                 "spider_adjust_logits: a history needs n_history and a stride of at most 2^31 - 2^14");
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
                     logits_stride, out_stride, history_stride, mask_stride, B, T, V, n_bias, ceil_div(V, adjust_piece(V))};
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  ProfScope ps(KC_ADJUST_LOGITS, st);
  // four logits at a time where every row starts on a 16-byte (bf16: 8-byte) boundary and has a multiple of 4
  const uintptr_t four = dtype == SPIDER_BF16 ? 7 : 15;
  const bool vec = V % 4 == 0 && logits_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(logits) & four) == 0 &&
                   (!out || (out_stride % 4 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0));
  if (dtype == SPIDER_BF16) {
    if (vec) launch_adjust<uint16_t, 4>(a, st);
    else launch_adjust<uint16_t, 1>(a, st);
  } else {
    if (vec) launch_adjust<float, 4>(a, st);
    else launch_adjust<float, 1>(a, st);
  }
  SPIDER_LAUNCHED("adjust_logits");
  if (next_out && a.pieces > 1) {
    adjust_join_kernel<<<(unsigned)(B * T), 64, 0, st>>>(a);
    SPIDER_LAUNCHED("adjust_join");
  }
  return SPIDER_OK;
}
