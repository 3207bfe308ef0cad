// Attention of a tree of drafted tokens over a key/value cache
// (spider_tree_attention) and the attention weight every slot receives.
//
//   s(r, j) = scale q_r . k_j,  o_r = sum_j softmax_j(s(r, .)) v_j
// over the slots j that row r = (node t, head h) sees: the context j < lens[b]
// and the nodes u = j - lens[b] whose bit is set in the node's mask.
#include <cmath>

#include "kernels.h"

namespace spider {
namespace {

constexpr int kTreeMaxNodes = 256;
constexpr int kTreeMaxDh = 256;

// What every kernel needs to know of one call.
struct TreeArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  const int32_t* lens;
  const int32_t* n_nodes;
  const uint64_t* mask;
  const float* w_in;
  float* w_out;
  float2* stat;  // [B][T][H] (largest score, 1 / sum of exponentials)
  int64_t qb, qt;         // strides of q, elements
  int64_t kvb, kvs, kvh;  // strides of k and v
  int B, T, H, Hkv, dh, cap;
  float scale;
};

// The filled slots and live nodes of sample b, clamped to the cache.
__device__ __forceinline__ int2 tree_extent(const TreeArgs& a, int b) {
  const int len = min(max(a.lens[b], 0), a.cap);
  const int nn = a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T;
  return make_int2(len, min(nn, a.cap - len));
}

// Whether node t of sample b sees node u.
__device__ __forceinline__ bool tree_sees(const TreeArgs& a, int b, int t, int u) {
  if (!a.mask) return u <= t;
  const int W = (a.T + 63) / 64;
  return (a.mask[((int64_t)b * a.T + t) * W + (u >> 6)] >> (u & 63)) & 1;
}

template <typename AT>
__device__ __forceinline__ float tree_load(const void* p, int64_t i) {
  if constexpr (sizeof(AT) == 4) return reinterpret_cast<const float*>(p)[i];
  else return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[i]);
}

template <typename AT>
__device__ __forceinline__ float tree_dot(const TreeArgs& a, const float* qs, int64_t kp) {
  float s = 0.f;
  for (int c = 0; c < a.dh; ++c) s = fmaf(qs[c], tree_load<AT>(a.k, kp + c), s);
  return s * a.scale;
}

// One block per (node, head, sample): the keys in pieces of 256, a thread per key
// for the scores and per channel for the values, with the running maximum and sum.
template <typename AT>
__global__ void __launch_bounds__(256) tree_rows_kernel(TreeArgs a) {
  __shared__ float qs[kTreeMaxDh];
  __shared__ float p[256];
  __shared__ float red[4];
  const int t = blockIdx.x / a.H, h = blockIdx.x - t * a.H, b = blockIdx.y;
  const int hk = h / (a.H / a.Hkv);
  const int tid = threadIdx.x, wave = tid >> 6;
  const int2 ext = tree_extent(a, b);
  if (t >= ext.y) return;
  const int n = ext.x + ext.y;
  const int64_t qp = b * a.qb + t * a.qt + (int64_t)h * a.dh;
  const int64_t kv = b * a.kvb + hk * a.kvh;
  if (tid < a.dh) qs[tid] = tree_load<AT>(a.q, qp + tid);
  __syncthreads();
  float top = -INFINITY, sum = 0.f, o = 0.f;
  for (int j0 = 0; j0 < n; j0 += 256) {
    const int j = j0 + tid;
    const bool sees = j < n && (j < ext.x || tree_sees(a, b, t, j - ext.x));
    const float s = sees ? tree_dot<AT>(a, qs, kv + j * a.kvs) : -INFINITY;
    const float wm = wave_max(s);
    if ((tid & 63) == 0) red[wave] = wm;
    __syncthreads();
    const float m = fmaxf(top, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float ms = m == -INFINITY ? 0.f : m;
    const float e = sees ? expf(s - ms) : 0.f;
    p[tid] = sees ? e : -1.f;  // -1: not seen, its value is not read
    __syncthreads();
    const float ws = wave_sum(e);
    if ((tid & 63) == 0) red[wave] = ws;
    __syncthreads();
    const float f = top == -INFINITY ? 0.f : expf(top - ms);
    sum = sum * f + ((red[0] + red[1]) + (red[2] + red[3]));
    o *= f;
    top = m;
    if (tid < a.dh)
      for (int i = 0; i < min(256, n - j0); ++i)
        if (p[i] != -1.f) o = fmaf(p[i], tree_load<AT>(a.v, kv + (j0 + i) * a.kvs + tid), o);
    __syncthreads();
  }
  const int64_t row = ((int64_t)b * a.T + t) * a.H + h;
  if (tid < a.dh) {
    const float x = sum == 0.f ? 0.f : o / sum;
    if constexpr (sizeof(AT) == 4) reinterpret_cast<float*>(a.out)[row * a.dh + tid] = x;
    else reinterpret_cast<uint16_t*>(a.out)[row * a.dh + tid] = f32_to_bf16_bits(x);
  }
  if (tid == 0 && a.stat) a.stat[row] = make_float2(top == -INFINITY ? 0.f : top, sum == 0.f ? 0.f : 1.f / sum);
}

// A thread per (slot, kv head, sample): the weight that all live rows of the head
// group give the slot, from the rows' final maximum and sum.
template <typename AT>
__global__ void __launch_bounds__(256) tree_weights_kernel(TreeArgs a) {
  const int j = blockIdx.x * 256 + threadIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const int2 ext = tree_extent(a, b);
  if (j >= ext.x + ext.y) return;
  const int G = a.H / a.Hkv;
  const int64_t kp = b * a.kvb + hk * a.kvh + j * a.kvs;
  const int64_t w = ((int64_t)b * a.Hkv + hk) * a.cap + j;
  float sum = 0.f;
  for (int t = 0; t < ext.y; ++t) {
    if (j >= ext.x && !tree_sees(a, b, t, j - ext.x)) continue;
    for (int g = 0; g < G; ++g) {
      const int h = hk * G + g;
      const int64_t qp = b * a.qb + t * a.qt + (int64_t)h * a.dh;
      float s = 0.f;
      for (int c = 0; c < a.dh; ++c) s = fmaf(tree_load<AT>(a.q, qp + c), tree_load<AT>(a.k, kp + c), s);
      const float2 st = a.stat[((int64_t)b * a.T + t) * a.H + h];
      sum += expf(s * a.scale - st.x) * st.y;
    }
  }
  a.w_out[w] = (j < ext.x && a.w_in ? a.w_in[w] : 0.f) + sum;
}

size_t tree_ws_bytes(int B, int T, int H, bool weights) {
  return weights ? align_up((size_t)B * T * H * sizeof(float2), 256) : 0;
}

template <typename AT>
spider_status run_tree(const TreeArgs& a, hipStream_t st) {
  {
    ProfScope ps(KC_TREE_ATTN, st);
    tree_rows_kernel<AT><<<dim3((unsigned)(a.T * a.H), (unsigned)a.B), 256, 0, st>>>(a);
    SPIDER_LAUNCHED("tree_rows");
  }
  if (a.w_out) {
    ProfScope ps(KC_TREE_WEIGHTS, st);
    tree_weights_kernel<AT><<<dim3((unsigned)ceil_div(a.cap, 256), (unsigned)a.Hkv, (unsigned)a.B), 256, 0, st>>>(a);
    SPIDER_LAUNCHED("tree_weights");
  }
  return SPIDER_OK;
}

bool tree_shape_ok(int B, int T, int H, int Hkv, int dh, int cap, spider_dtype dtype) {
  return B >= 1 && B <= 65535 && T >= 1 && T <= kTreeMaxNodes && H >= 1 && H <= 65535 && Hkv >= 1 && H % Hkv == 0 &&
         dh >= 1 && dh <= kTreeMaxDh && cap >= 1 && (dtype == SPIDER_BF16 || dtype == SPIDER_F32);
}

}  // namespace
}  // namespace spider

using namespace spider;

extern "C" size_t spider_tree_attention_workspace_size(int B, int T, int H, int Hkv, int dh, int cap,
                                                       spider_dtype dtype, int weights) {
  if (!tree_shape_ok(B, T, H, Hkv, dh, cap, dtype)) return 0;
  return tree_ws_bytes(B, T, H, weights != 0);
}

extern "C" spider_status spider_tree_attention(int B, int T, int H, int Hkv, int dh, const void* q,
                                               int64_t q_stride_b, int64_t q_stride_t, const void* k, const void* v,
                                               int64_t kv_stride_b, int64_t kv_stride_s, int64_t kv_stride_h, int cap,
                                               const int32_t* lens, const int32_t* n_nodes, const uint64_t* tree_mask,
                                               spider_dtype dtype, float scale, void* out, const float* weights_in,
                                               float* weights_out, void* workspace, size_t workspace_bytes,
                                               spider_stream stream) {
  clear_error();
  SPIDER_REQUIRE(q && k && v && lens && out, SPIDER_ERR_INVALID_ARG, "spider_tree_attention: null pointer");
  SPIDER_REQUIRE(dtype == SPIDER_BF16 || dtype == SPIDER_F32, SPIDER_ERR_INVALID_ARG,
                 "spider_tree_attention: bad dtype");
  SPIDER_REQUIRE(!weights_in || weights_out, SPIDER_ERR_INVALID_ARG,
                 "spider_tree_attention: weights_in without weights_out");
  SPIDER_REQUIRE(B >= 1 && T >= 1 && H >= 1 && Hkv >= 1 && dh >= 1 && cap >= 1, SPIDER_ERR_INVALID_ARG,
                 "spider_tree_attention: sizes must be positive");
  SPIDER_REQUIRE(H % Hkv == 0, SPIDER_ERR_SHAPE, "spider_tree_attention: %d heads over %d kv heads", H, Hkv);
  SPIDER_REQUIRE(T <= kTreeMaxNodes && dh <= kTreeMaxDh && B <= 65535 && H <= 65535, SPIDER_ERR_UNSUPPORTED,
                 "spider_tree_attention: T <= %d, dh <= %d, B and H <= 65535", kTreeMaxNodes, kTreeMaxDh);
  const int64_t per16 = dtype == SPIDER_BF16 ? 8 : 4;
  SPIDER_REQUIRE(dh % per16 == 0, SPIDER_ERR_UNSUPPORTED, "spider_tree_attention: dh must be a multiple of 16 bytes");
  SPIDER_REQUIRE(q_stride_b % per16 == 0 && q_stride_t % per16 == 0 && kv_stride_b % per16 == 0 &&
                     kv_stride_s % per16 == 0 && kv_stride_h % per16 == 0,
                 SPIDER_ERR_INVALID_ARG, "spider_tree_attention: strides must be multiples of 16 bytes");
  SPIDER_REQUIRE(q_stride_b >= 0 && q_stride_t >= 0 && kv_stride_b >= 0 && kv_stride_s >= 0 && kv_stride_h >= 0,
                 SPIDER_ERR_INVALID_ARG, "spider_tree_attention: negative stride");
  const uintptr_t bits = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k) |
                         reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(out);
  SPIDER_REQUIRE(bits % 16 == 0, SPIDER_ERR_INVALID_ARG, "spider_tree_attention: q, k, v and out must be 16-byte aligned");
  const size_t need = tree_ws_bytes(B, T, H, weights_out != nullptr);
  SPIDER_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), SPIDER_ERR_WORKSPACE,
                 "spider_tree_attention: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : 0);
  SPIDER_REQUIRE(need == 0 || reinterpret_cast<uintptr_t>(workspace) % 256 == 0, SPIDER_ERR_INVALID_ARG,
                 "spider_tree_attention: workspace must be 256-byte aligned");
  TreeArgs a{q, k, v, out, lens, n_nodes, tree_mask, weights_in, weights_out, reinterpret_cast<float2*>(workspace),
             q_stride_b, q_stride_t, kv_stride_b, kv_stride_s, kv_stride_h, B, T, H, Hkv, dh, cap, scale};
  if (!weights_out) a.stat = nullptr;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  return dtype == SPIDER_BF16 ? run_tree<uint16_t>(a, st) : run_tree<float>(a, st);
}
