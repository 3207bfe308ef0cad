// Eviction from a key/value cache by accumulated attention weight:
// spider_cache_select chooses the slots a cache keeps, spider_cache_compact
// moves their keys, values and weights to the front.
#include <cmath>

#include "kernels.h"

namespace spider {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;

struct SelectArgs {
  const float* w;  // [L][B][Hkv][cap]
  const int32_t* lens;
  int32_t* idx;    // [L][B][G][keep]
  int32_t* len_out;
  int L, B, Hkv, G, cap, keep, n_first, n_last;
};

// Order of slot j of one row of n slots: the slots that are always kept above every
// weight, NaN like -inf, -0 like +0.
__device__ __forceinline__ uint32_t slot_key(const SelectArgs& a, const float* w, int j, int n) {
  if (j < a.n_first || j >= n - a.n_last) return 0xFFFFFFFFu;
  float x;
  if (a.G == a.Hkv) {
    x = w[j];
  } else {
    double s = 0.0;  // over the heads in order
    for (int h = 0; h < a.Hkv; ++h) s += (double)w[(int64_t)h * a.cap + j];
    x = (float)s;
  }
  return float_order_key(x != x ? -INFINITY : x);
}

// One block per (layer, sample, head group): the keep-th largest key byte by byte
// from a histogram of the keys that share the bytes found so far, then the kept
// slots in ascending order.
__global__ void __launch_bounds__(kSelThreads) cache_select_kernel(SelectArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];  // byte, keys still wanted within it
  __shared__ uint2 tot[kSelWaves];
  const int row = blockIdx.x;  // (l * B + b) * G + g
  const int g = row % a.G, lb = row / a.G, b = lb % a.B;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.lens[b], 0), a.cap);
  const float* w = a.w + ((int64_t)lb * a.Hkv + g) * a.cap;
  int32_t* idx = a.idx + (int64_t)row * a.keep;
  if (lb == b && g == 0 && tid == 0) a.len_out[b] = min(n, a.keep);
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += kSelThreads) idx[i] = i < n ? i : -1;
    return;
  }
  uint32_t prefix = 0, want = (uint32_t)a.keep;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += kSelThreads) {
      const uint32_t k = slot_key(a, w, j, n);
      if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t left = want;
      int v = 255;
      while (hist[v] < left) left -= hist[v--];
      found[0] = (uint32_t)v;
      found[1] = left;
    }
    __syncthreads();
    prefix = (prefix << 8) | found[0];
    want = found[1];
    __syncthreads();
  }
  // all slots above the key `prefix`, and the first `want` slots that equal it
  uint32_t above = 0, equal = 0;
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    const uint32_t k = j < n ? slot_key(a, w, j, n) : 0u;
    const bool gt = j < n && k > prefix, eq = j < n && k == prefix;
    const uint64_t mg = __ballot(gt), me = __ballot(eq);
    if (lane == 0) tot[wave] = make_uint2(__popcll(mg), __popcll(me));
    __syncthreads();
    uint32_t ga = above, ea = equal;
    for (int v = 0; v < kSelWaves; ++v) {
      const uint2 c = tot[v];
      above += c.x;
      equal += c.y;
      if (v < wave) {
        ga += c.x;
        ea += c.y;
      }
    }
    const uint64_t below = (1ull << lane) - 1ull;
    ga += __popcll(mg & below);
    ea += __popcll(me & below);
    if (gt || (eq && ea < want)) idx[ga + min(ea, want)] = j;
    __syncthreads();
  }
}

struct CompactArgs {
  const char* in[2];  // keys, values
  char* out[2];
  const float* w_in;  // [L][B][Hkv][cap_in] or null
  float* w_out;
  const int32_t* idx;    // [idx_layers][B][idx_heads][n_max]
  const int32_t* count;  // [B] or null
  const int32_t* base;   // [B] or null
  int64_t il, ib, is, ih, ol, ob, os, oh;  // strides, bytes
  int L, B, Hkv, nv, cap_in, cap_out, n_max, idx_layers, idx_heads;
};

// Where entry i of (l, b, h) comes from and goes to; false where there is none.
struct CompactRow {
  const int32_t* idx;
  int n, base;
};
__device__ __forceinline__ CompactRow compact_row(const CompactArgs& a, int l, int b, int h) {
  const int64_t r = ((int64_t)(a.idx_layers == 1 ? 0 : l) * a.B + b) * a.idx_heads + (a.idx_heads == 1 ? 0 : h);
  return CompactRow{a.idx + r * a.n_max, a.count ? min(max(a.count[b], 0), a.n_max) : a.n_max, a.base ? a.base[b] : 0};
}
__device__ __forceinline__ bool compact_entry(const CompactArgs& a, const CompactRow& r, int i, int& src, int& dst) {
  if (i >= r.n) return false;
  const int x = r.idx[i];
  const int64_t s = (int64_t)r.base + x, d = (int64_t)r.base + i;
  src = (int)s;
  dst = (int)d;
  return x >= 0 && r.base >= 0 && s < a.cap_in && d < a.cap_out;
}

// Into another cache: a thread per 16-byte piece of an entry, its key and its value.
__global__ void __launch_bounds__(256) cache_copy_kernel(CompactArgs a) {
  const int lbh = blockIdx.y, h = lbh % a.Hkv, b = lbh / a.Hkv % a.B, l = lbh / a.Hkv / a.B;
  const CompactRow r = compact_row(a, l, b, h);
  const int per = 256 / a.nv, c = threadIdx.x % a.nv, e = threadIdx.x / a.nv;
  const int i = blockIdx.x * per + e;
  int src, dst;
  if (e >= per || !compact_entry(a, r, i, src, dst)) return;
  const int64_t ip = l * a.il + b * a.ib + src * a.is + h * a.ih + 16 * c;
  const int64_t op = l * a.ol + b * a.ob + dst * a.os + h * a.oh + 16 * c;
  const u32x4 k = *reinterpret_cast<const u32x4*>(a.in[0] + ip), v = *reinterpret_cast<const u32x4*>(a.in[1] + ip);
  *reinterpret_cast<u32x4*>(a.out[0] + op) = k;
  *reinterpret_cast<u32x4*>(a.out[1] + op) = v;
  if (a.w_out && c == 0) a.w_out[(int64_t)lbh * a.cap_out + dst] = a.w_in[(int64_t)lbh * a.cap_in + src];
}

// In place: one block per (layer, sample, head, kind) walks its entries in ascending
// order.  An entry never comes from below the slot it goes to, so no later entry reads
// what an earlier piece has written; within a piece every read precedes every write.
__global__ void __launch_bounds__(256) cache_move_kernel(CompactArgs a) {
  const int lbh = blockIdx.x, h = lbh % a.Hkv, b = lbh / a.Hkv % a.B, l = lbh / a.Hkv / a.B;
  const int kind = blockIdx.y;
  const CompactRow r = compact_row(a, l, b, h);
  if (kind == 2) {
    const float* in = a.w_in + (int64_t)lbh * a.cap_in;
    float* out = a.w_out + (int64_t)lbh * a.cap_out;
    for (int i0 = 0; i0 < r.n; i0 += 256) {
      int src, dst;
      const bool on = compact_entry(a, r, i0 + threadIdx.x, src, dst) && src != dst;
      const float x = on ? in[src] : 0.f;
      __syncthreads();
      if (on) out[dst] = x;
      __syncthreads();
    }
    return;
  }
  const int per = 256 / a.nv, c = threadIdx.x % a.nv, e = threadIdx.x / a.nv;
  const char* in = a.in[kind] + l * a.il + b * a.ib + h * a.ih + 16 * c;
  char* out = a.out[kind] + l * a.ol + b * a.ob + h * a.oh + 16 * c;
  for (int i0 = 0; i0 < r.n; i0 += per) {
    int src, dst;
    const bool on = e < per && compact_entry(a, r, i0 + e, src, dst) && src != dst;
    u32x4 x = {0, 0, 0, 0};
    if (on) x = *reinterpret_cast<const u32x4*>(in + src * a.is);
    __syncthreads();
    if (on) *reinterpret_cast<u32x4*>(out + dst * a.os) = x;
    __syncthreads();
  }
}

}  // namespace
}  // namespace spider

using namespace spider;

extern "C" spider_status spider_cache_select(int L, int B, int Hkv, int cap, const float* weights, const int32_t* lens,
                                             int keep, int n_first, int n_last, int shared, int32_t* idx_out,
                                             int32_t* len_out, spider_stream stream) {
  clear_error();
  SPIDER_REQUIRE(weights && lens && idx_out && len_out, SPIDER_ERR_INVALID_ARG, "spider_cache_select: null pointer");
  SPIDER_REQUIRE(L >= 1 && B >= 1 && Hkv >= 1 && cap >= 1, SPIDER_ERR_INVALID_ARG,
                 "spider_cache_select: sizes must be positive");
  SPIDER_REQUIRE(keep >= 1 && n_first >= 0 && n_last >= 0, SPIDER_ERR_INVALID_ARG,
                 "spider_cache_select: keep >= 1, n_first and n_last >= 0");
  SPIDER_REQUIRE(shared == 0 || shared == 1, SPIDER_ERR_INVALID_ARG, "spider_cache_select: shared must be 0 or 1");
  SPIDER_REQUIRE((int64_t)n_first + n_last <= keep, SPIDER_ERR_SHAPE,
                 "spider_cache_select: n_first + n_last = %lld exceed keep = %d", (long long)n_first + n_last, keep);
  SPIDER_REQUIRE(keep <= cap, SPIDER_ERR_SHAPE, "spider_cache_select: keep = %d exceeds cap = %d", keep, cap);
  const int G = shared ? 1 : Hkv;
  SPIDER_REQUIRE((int64_t)L * B * G <= 0x7fffffff, SPIDER_ERR_UNSUPPORTED, "spider_cache_select: too many rows");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  ProfScope ps(KC_CACHE_SELECT, st);
  const SelectArgs a{weights, lens, idx_out, len_out, L, B, Hkv, G, cap, keep, n_first, n_last};
  cache_select_kernel<<<(unsigned)(L * B * G), kSelThreads, 0, st>>>(a);
  SPIDER_LAUNCHED("cache_select");
  return SPIDER_OK;
}

extern "C" spider_status spider_cache_compact(int L, int B, int Hkv, int dh, spider_dtype dtype, const void* k_in,
                                              const void* v_in, const int64_t in_strides[4], int cap_in, void* k_out,
                                              void* v_out, const int64_t out_strides[4], int cap_out,
                                              const int32_t* idx, int idx_layers, int idx_heads, int n_max,
                                              const int32_t* count, const int32_t* base, const float* weights_in,
                                              float* weights_out, spider_stream stream) {
  clear_error();
  SPIDER_REQUIRE(k_in && v_in && k_out && v_out && in_strides && out_strides && (idx || n_max == 0), SPIDER_ERR_INVALID_ARG,
                 "spider_cache_compact: null pointer");
  SPIDER_REQUIRE(dtype == SPIDER_BF16 || dtype == SPIDER_F32, SPIDER_ERR_INVALID_ARG,
                 "spider_cache_compact: bad dtype");
  SPIDER_REQUIRE(L >= 1 && B >= 1 && Hkv >= 1 && dh >= 1 && cap_in >= 1 && cap_out >= 1 && n_max >= 0,
                 SPIDER_ERR_INVALID_ARG, "spider_cache_compact: sizes must be positive");
  SPIDER_REQUIRE((idx_layers == 1 || idx_layers == L) && (idx_heads == 1 || idx_heads == Hkv), SPIDER_ERR_SHAPE,
                 "spider_cache_compact: idx has %d layers and %d heads, 1 or %d and 1 or %d wanted", idx_layers,
                 idx_heads, L, Hkv);
  SPIDER_REQUIRE((weights_in != nullptr) == (weights_out != nullptr), SPIDER_ERR_INVALID_ARG,
                 "spider_cache_compact: weights_in and weights_out go together");
  const int es = dtype == SPIDER_BF16 ? 2 : 4;
  SPIDER_REQUIRE(dh * es % 16 == 0 && dh <= 256, SPIDER_ERR_UNSUPPORTED,
                 "spider_cache_compact: dh must be a multiple of 16 bytes and at most 256");
  const uintptr_t bits = reinterpret_cast<uintptr_t>(k_in) | reinterpret_cast<uintptr_t>(v_in) |
                         reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out);
  SPIDER_REQUIRE(bits % 16 == 0, SPIDER_ERR_INVALID_ARG, "spider_cache_compact: the caches must be 16-byte aligned");
  bool same = cap_in == cap_out;
  for (int i = 0; i < 4; ++i) {
    SPIDER_REQUIRE(in_strides[i] >= 0 && out_strides[i] >= 0 && in_strides[i] * es % 16 == 0 &&
                       out_strides[i] * es % 16 == 0,
                   SPIDER_ERR_INVALID_ARG, "spider_cache_compact: strides must be multiples of 16 bytes");
    same = same && in_strides[i] == out_strides[i];
  }
  const bool inplace = k_in == k_out;
  SPIDER_REQUIRE(inplace == (v_in == v_out) && (!weights_in || inplace == (weights_in == weights_out)),
                 SPIDER_ERR_INVALID_ARG, "spider_cache_compact: keys, values and weights all move in place or none");
  SPIDER_REQUIRE(!inplace || same, SPIDER_ERR_SHAPE,
                 "spider_cache_compact: in place, the strides and capacities of both sides must be the same");
  SPIDER_REQUIRE((int64_t)L * B * Hkv <= 65535, SPIDER_ERR_UNSUPPORTED,
                 "spider_cache_compact: L * B * Hkv must be at most 65535");
  if (n_max == 0) return SPIDER_OK;
  CompactArgs a{};
  a.in[0] = reinterpret_cast<const char*>(k_in);
  a.in[1] = reinterpret_cast<const char*>(v_in);
  a.out[0] = reinterpret_cast<char*>(k_out);
  a.out[1] = reinterpret_cast<char*>(v_out);
  a.w_in = weights_in;
  a.w_out = weights_out;
  a.idx = idx;
  a.count = count;
  a.base = base;
  a.il = in_strides[0] * es, a.ib = in_strides[1] * es, a.is = in_strides[2] * es, a.ih = in_strides[3] * es;
  a.ol = out_strides[0] * es, a.ob = out_strides[1] * es, a.os = out_strides[2] * es, a.oh = out_strides[3] * es;
  a.L = L, a.B = B, a.Hkv = Hkv, a.nv = dh * es / 16;
  a.cap_in = cap_in, a.cap_out = cap_out, a.n_max = n_max, a.idx_layers = idx_layers, a.idx_heads = idx_heads;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  ProfScope ps(KC_CACHE_COMPACT, st);
  const unsigned rows = (unsigned)(L * B * Hkv);
  if (inplace)
    cache_move_kernel<<<dim3(rows, weights_in ? 3 : 2), 256, 0, st>>>(a);
  else
    cache_copy_kernel<<<dim3((unsigned)ceil_div(n_max, 256 / a.nv), rows), 256, 0, st>>>(a);
  SPIDER_LAUNCHED("cache_compact");
  return SPIDER_OK;
}
