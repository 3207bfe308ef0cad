// Eviction from a key/value cache by accumulated attention weight:
// spider_cache_select chooses the slots a cache keeps, spider_cache_compact
// moves their keys, values and weights to the front.
// Measured on one MI355X: 1024 rows of 2944 slots, 576 kept, selection 19 us, copy of
// their keys and values (bf16 of 128) into another cache 119 us (5.1 TB/s); 64 rows of
// 65536, 16384 kept, 58 and 209 us (5.1 TB/s).
#include <cmath>

#include "kernels.h"

namespace spider {
namespace {

struct SelectArgs {
  const float* w;  // [L][B][Hkv][cap]
  const int32_t* lens;
  int32_t* idx;    // [L][B][G][keep]
  int32_t* len_out;
  int L, B, Hkv, G, cap, keep, n_first, n_last;
};

// Weight of slot j: its own, or added over the heads in order.
__device__ __forceinline__ float slot_weight(const SelectArgs& a, const float* w, int j) {
  if (a.G == a.Hkv) return w[j];
  double s = 0.0;
  for (int h0 = 0; h0 < a.Hkv; h0 += 4) {  // four loads in flight
    float x[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) x[h] = w[(int64_t)min(h0 + h, a.Hkv - 1) * a.cap + j];
#pragma unroll
    for (int h = 0; h < 4; ++h)
      if (h0 + h < a.Hkv) s += (double)x[h];
  }
  return (float)s;
}

// Order of slot j of a row of n slots: the slots that are always kept above every
// weight, NaN like -inf (0x007FFFFF), -0 like +0; 0 past the last slot.
__device__ __forceinline__ uint32_t slot_key(const SelectArgs& a, float x, int j, int n) {
  const uint32_t k = j < a.n_first || j >= n - a.n_last ? 0xFFFFFFFFu : float_order_key(x != x ? -INFINITY : x);
  return j < n ? k : 0u;
}

// Sum over this lane and the lower ones: within rows of 16 lanes, then across them.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);  // row_shr:1, 2, 4, 8
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1 and 3
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2 and 3
  return v;
}

constexpr int kSelBits = 11;  // of a key per pass: 32 = 11 + 11 + 10
constexpr int kSelBuckets = 1 << kSelBits;

// The bucket of the want-th largest key and its place within the bucket: lane l sums 32
// buckets, the highest first, then 32 lanes look at those of the lane where the count is
// reached.  One wave; found = (bucket, keys still wanted within it).
__device__ __forceinline__ void find_bucket(const uint32_t* hist, uint32_t want, uint32_t* found) {
  const int lane = threadIdx.x & 63;
  uint32_t s = 0;
  const int top = kSelBuckets - 1 - 32 * lane;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += hist[top - ((i + lane) & 31)];
  const uint32_t up = wave_prefix(s);
  const int at = __ffsll((unsigned long long)__ballot(up >= want)) - 1;
  const uint32_t left = want - (uint32_t)__builtin_amdgcn_readlane((int)(up - s), at);
  const uint32_t c = lane < 32 ? hist[kSelBuckets - 1 - 32 * at - lane] : 0u;
  const uint32_t in = wave_prefix(c);
  const int v = __ffsll((unsigned long long)__ballot(lane < 32 && in >= left)) - 1;
  if (lane == v) {
    found[0] = (uint32_t)(kSelBuckets - 1 - 32 * at - lane);
    found[1] = left - (in - c);
  }
}

// Counts a key's bucket (on: of the lanes that count): one add for the lanes that share the
// first lane's bucket, since weights crowd in few exponents and often in one value.
__device__ __forceinline__ void count_bucket(uint32_t* hist, uint32_t bucket, bool on) {
  const uint64_t active = __ballot(on);
  if (active == 0) return;
  const int lane = threadIdx.x & 63, leader = __ffsll((unsigned long long)active) - 1;
  const bool same = on && bucket == (uint32_t)__builtin_amdgcn_readlane((int)bucket, leader);
  const uint64_t group = __ballot(same);
  if (lane == leader) atomicAdd(&hist[bucket], (uint32_t)__popcll(group));
  else if (on && !same) atomicAdd(&hist[bucket], 1u);
}

// One block per (layer, sample, head group): the keep-th largest key by a histogram of
// its upper bits, then of the next bits of the keys that share those, then of the rest;
// then the kept slots in ascending order.  Wave w owns 64 * NV consecutive slots, so that
// after one exchange of counts every wave writes its slots without a barrier.  The keys
// stay in registers (NV > 0, up to 64 per lane: n <= THREADS * NV); longer rows are read
// again in each pass (NV = 0).
// Bound by the barriers and the LDS atomics of its passes (a row is read once).
template <int THREADS, int NV>
__global__ void __launch_bounds__(THREADS) cache_select_kernel(SelectArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ uint32_t hist[kSelBuckets];
  __shared__ uint32_t found[2];  // bucket, keys still wanted within it
  __shared__ uint2 tot[WAVES];
  const int row = blockIdx.x;  // (l * B + b) * G + g
  const int g = row % a.G, lb = row / a.G, b = lb % a.B;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.lens[b], 0), a.cap);
  const float* w = a.w + ((int64_t)lb * a.Hkv + g) * a.cap;
  int32_t* idx = a.idx + (int64_t)row * a.keep;
  if (lb == b && g == 0 && tid == 0) a.len_out[b] = min(n, a.keep);
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += THREADS) idx[i] = i < n ? i : -1;
    return;
  }
  const int nv = NV ? NV : (n + THREADS - 1) / THREADS;  // 64-slot pieces of a wave
  int j0 = wave * nv * 64 + lane;
  uint32_t keys[NV ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int i0 = 0; i0 < NV; i0 += 16) {  // 16 loads in flight
#pragma unroll
      for (int i = i0; i < i0 + 16; ++i) keys[i] = __float_as_uint(slot_weight(a, w, min(j0 + 64 * i, n - 1)));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = i0; i < i0 + 16; ++i) keys[i] = slot_key(a, __uint_as_float(keys[i]), j0 + 64 * i, n);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // f(key, slot) for every slot of the wave in ascending pieces
  auto each = [&](auto&& f) {
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        f(keys[i], j0 + 64 * i);
      }
    } else {
      for (int i0 = 0; i0 < nv; i0 += 8) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = slot_weight(a, w, min(j0 + 64 * (i0 + i), n - 1));
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i0 + i < nv) f(slot_key(a, x[i], j0 + 64 * (i0 + i), n), j0 + 64 * (i0 + i));
      }
    }
  };
  uint32_t prefix = 0, want = (uint32_t)a.keep;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < kSelBuckets; i += THREADS) hist[i] = 0;
    __syncthreads();
    each([&](uint32_t k, int) {
      // (in the first pass all, also the zeros past the last slot: no search goes down to their bucket)
      const bool on = (k >> (shift + bits - 1)) >> 1 == prefix;
      count_bucket(hist, (k >> shift) & ((1u << bits) - 1u), on);
    });
    __syncthreads();
    if (wave == 0) find_bucket(hist, want, found);
    __syncthreads();
    prefix = __builtin_amdgcn_readfirstlane((prefix << bits) | found[0]);
    want = __builtin_amdgcn_readfirstlane(found[1]);
  }
  // all slots above the key `prefix`, and the first `want` slots that equal it
  uint32_t gt = 0, eq = 0;
  each([&](uint32_t k, int) {
    gt += __popcll(__ballot(k > prefix));
    eq += __popcll(__ballot(k == prefix));
  });
  // the comparisons and slots below are made again, not kept in 3 * NV registers
  asm volatile("" : "+s"(prefix), "+v"(j0));
  if (lane == 0) tot[wave] = make_uint2(gt, eq);
  __syncthreads();
  gt = eq = 0;
  for (int v = 0; v < wave; ++v) {
    gt += tot[v].x;
    eq += tot[v].y;
  }
  const uint64_t below = (1ull << lane) - 1ull;
  each([&](uint32_t k, int j) {
    const uint64_t mg = __ballot(k > prefix), me = __ballot(k == prefix);
    const uint32_t ga = gt + __popcll(mg & below), ea = eq + __popcll(me & below);
    if (k > prefix || (k == prefix && ea < want)) idx[ga + min(ea, want)] = j;
    gt += __popcll(mg);
    eq += __popcll(me);
  });
}

// Long rows, few of them: the same selection with a block per chunk of 8192 slots, in four
// launches.  Every launch adds up the chunks' histograms of the one before (the same in all
// blocks of a row), and counts its own chunk's next bits:
//   1 keys (added over the heads here, once) and their upper 11 bits
//   2 the bucket of the keep-th key; the next 11 bits of its keys
//   3 again, the last 10 bits
//   4 the key itself; where the chunk's slots go, and the slots
constexpr int kChunk = 8192, kChunkThreads = 512, kChunkKeys = kChunk / kChunkThreads;
struct ChunkWs {
  uint32_t* keys;   // [rows][chunks][kChunk]
  uint32_t* hist;   // [3][rows][chunks][kSelBuckets]
  uint32_t* found;  // [2][rows][2] bucket and keys wanted after launches 2 and 3
  uint32_t* above;  // [2][rows][chunks] keys of the chunk above the bucket of its launch
};

// Sum over the block, in every thread.
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t* cell) {
  if (threadIdx.x == 0) *cell = 0;
  __syncthreads();
  const int x = wave_sum_int((int)v);
  if ((threadIdx.x & 63) == 0) atomicAdd(cell, (uint32_t)x);
  __syncthreads();
  return *cell;
}

template <int PHASE>
__global__ void __launch_bounds__(kChunkThreads) cache_select_chunk_kernel(SelectArgs a, ChunkWs ws, int chunks) {
  constexpr int WAVES = kChunkThreads / 64;
  __shared__ uint32_t hist[kSelBuckets];
  __shared__ uint32_t found[2], cell;
  __shared__ uint2 tot[WAVES];
  const int rows = a.L * a.B * a.G;
  const int row = blockIdx.x / chunks, ch = blockIdx.x % chunks;  // row = (l * B + b) * G + g
  const int g = row % a.G, lb = row / a.G, b = lb % a.B;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.lens[b], 0), a.cap);
  int32_t* idx = a.idx + (int64_t)row * a.keep;
  if (PHASE == 1 && lb == b && g == 0 && ch == 0 && tid == 0) a.len_out[b] = min(n, a.keep);
  if (n <= a.keep) {
    if (PHASE == 1)
      for (int i = ch * kChunk + tid; i < min(a.keep, (ch + 1) * kChunk); i += kChunkThreads) idx[i] = i < n ? i : -1;
    return;
  }
  if (ch * kChunk >= n) return;
  const int used = (n + kChunk - 1) / kChunk;
  uint32_t* kp = ws.keys + ((int64_t)row * chunks + ch) * kChunk;
  const int c0 = wave * (kChunk / WAVES) + lane;  // the wave's consecutive slots of the chunk
  uint32_t keys[kChunkKeys];
  if (PHASE == 1) {
    const float* w = a.w + ((int64_t)lb * a.Hkv + g) * a.cap;
    float x[kChunkKeys];
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i) x[i] = slot_weight(a, w, min(ch * kChunk + c0 + 64 * i, n - 1));
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i) keys[i] = slot_key(a, x[i], ch * kChunk + c0 + 64 * i, n);
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i) kp[c0 + 64 * i] = keys[i];
  } else {
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i) keys[i] = kp[c0 + 64 * i];
  }
  auto hist_of = [&](int level, int c) {
    return ws.hist + (((int64_t)level * rows + row) * chunks + c) * kSelBuckets;
  };
  uint32_t prefix = 0, want = (uint32_t)a.keep;
  if (PHASE > 1) {
    uint32_t own[kSelBuckets / kChunkThreads];
#pragma unroll
    for (int i = 0; i < kSelBuckets / kChunkThreads; ++i) {
      const int v = tid + i * kChunkThreads;
      uint32_t sum = 0;
      for (int c = 0; c < used; ++c) sum += hist_of(PHASE - 2, c)[v];
      hist[v] = sum;
      own[i] = hist_of(PHASE - 2, ch)[v];
    }
    if (PHASE > 2) {
      prefix = ws.found[row * 2];
      want = ws.found[row * 2 + 1];
    }
    if (PHASE > 3) {
      prefix = (prefix << 11) | ws.found[(rows + row) * 2];
      want = ws.found[(rows + row) * 2 + 1];
    }
    __syncthreads();
    if (wave == 0) find_bucket(hist, want, found);
    __syncthreads();
    const uint32_t bucket = found[0];
    want = found[1];
    if (PHASE < 4) {
      uint32_t up = 0;
#pragma unroll
      for (int i = 0; i < kSelBuckets / kChunkThreads; ++i) up += tid + i * kChunkThreads > (int)bucket ? own[i] : 0u;
      up = block_sum(up, &cell);
      if (tid == 0) ws.above[((int64_t)(PHASE - 2) * rows + row) * chunks + ch] = up;
      if (tid == 0 && ch == 0) {
        ws.found[((PHASE - 2) * rows + row) * 2] = bucket;
        ws.found[((PHASE - 2) * rows + row) * 2 + 1] = want;
      }
    }
    prefix = __builtin_amdgcn_readfirstlane((prefix << (PHASE == 4 ? 10 : 11)) | bucket);
  }
  if (PHASE < 4) {
    constexpr int shift = PHASE == 1 ? 21 : (PHASE == 2 ? 10 : 0), bits = PHASE == 3 ? 10 : 11;
    __syncthreads();
    for (int i = tid; i < kSelBuckets; i += kChunkThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i)
      count_bucket(hist, (keys[i] >> shift) & ((1u << bits) - 1u), (keys[i] >> (shift + bits - 1)) >> 1 == prefix);
    __syncthreads();
    uint32_t* h = hist_of(PHASE - 1, ch);
    for (int i = tid; i < kSelBuckets; i += kChunkThreads) h[i] = hist[i];
    return;
  }
  // the slots above the key and equal to it in the chunks before, then in the waves before
  uint32_t gt = 0, eq = 0;
  for (int c = 0; c < ch; ++c) {
    const uint32_t* h = hist_of(2, c);
    for (int v = tid; v < 1024; v += kChunkThreads) {
      const uint32_t x = h[v];
      gt += v > (int)found[0] ? x : 0u;
      eq += v == (int)found[0] ? x : 0u;
    }
    if (tid < 2) gt += ws.above[((int64_t)tid * rows + row) * chunks + c];
  }
  gt = block_sum(gt, &cell);
  __syncthreads();
  eq = block_sum(eq, &cell);
  uint32_t wg = 0, we = 0;
#pragma unroll
  for (int i = 0; i < kChunkKeys; ++i) {
    wg += __popcll(__ballot(keys[i] > prefix));
    we += __popcll(__ballot(keys[i] == prefix));
  }
  if (lane == 0) tot[wave] = make_uint2(wg, we);
  __syncthreads();
  for (int v = 0; v < wave; ++v) {
    gt += tot[v].x;
    eq += tot[v].y;
  }
  const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
  for (int i = 0; i < kChunkKeys; ++i) {
    const uint32_t k = keys[i];
    const uint64_t mg = __ballot(k > prefix), me = __ballot(k == prefix);
    const uint32_t ga = gt + __popcll(mg & below), ea = eq + __popcll(me & below);
    if (k > prefix || (k == prefix && ea < want)) idx[ga + min(ea, want)] = ch * kChunk + c0 + 64 * i;
    gt += __popcll(mg);
    eq += __popcll(me);
  }
}

// Rows in chunks, or a block per row: chunks while they leave CUs idle, and a little longer
// where a block per row would also add up the heads alone.  Measured with the move of the
// slots, chunks / rows, us: 50 rows of 32329 39 / 47; 64 of 65536 270 / 263; 256 of 32000
// 89 / 63; 8 of 9000 29 / 18; 12 rows of 29725 over 8 heads 52 / 97.
bool select_in_chunks(int64_t rows, int cap, bool summed) {
  return cap > (summed ? kChunk : 2 * kChunk) && rows * ceil_div(cap, kChunk) <= (summed ? 512 : 256);
}

size_t select_layout(int64_t rows, int cap, bool summed, char* base, ChunkWs* ws) {
  if (!select_in_chunks(rows, cap, summed)) return 0;
  const size_t chunks = ceil_div(cap, kChunk);
  size_t off = 0;
  auto take = [&](size_t n) {
    char* p = base ? base + off : nullptr;
    off = align_up(off + n * sizeof(uint32_t), 256);
    return reinterpret_cast<uint32_t*>(p);
  };
  ChunkWs w;
  w.keys = take(rows * chunks * kChunk);
  w.hist = take(3 * rows * chunks * kSelBuckets);
  w.found = take(4 * rows);
  w.above = take(2 * rows * chunks);
  if (ws) *ws = w;
  return off;
}

bool select_shape_ok(int L, int B, int Hkv, int cap, int shared) {
  return L >= 1 && B >= 1 && Hkv >= 1 && cap >= 1 && cap <= (1 << 30) && (shared == 0 || shared == 1) &&
         (int64_t)L * B * (shared ? 1 : Hkv) < (1 << 22);
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

// In place: blocks of a (layer, sample, head) each own cw 16-byte columns of the keys or of
// the values (kind 0, 1), or the weights (2), and walk the entries in ascending order, kMove
// per thread at a time.  An entry never comes from below the slot it goes to, so what a
// piece of entries writes lies below all that later pieces read; within a piece every read
// has returned before the first write, hence the wait and the barrier between them.
constexpr int kMove = 8;
__global__ void __launch_bounds__(256) cache_move_kernel(CompactArgs a, int cw) {
  const int lbh = blockIdx.x, h = lbh % a.Hkv, b = lbh / a.Hkv % a.B, l = lbh / a.Hkv / a.B;
  const int columns = (a.nv + cw - 1) / cw, kind = blockIdx.y / columns;
  const CompactRow r = compact_row(a, l, b, h);
  int src[kMove], dst[kMove];
  bool on[kMove];
  if (kind == 2) {
    if (blockIdx.y % columns != 0) return;
    const float* in = a.w_in + (int64_t)lbh * a.cap_in;
    float* out = a.w_out + (int64_t)lbh * a.cap_out;
    for (int i0 = 0; i0 < r.n; i0 += 256 * kMove) {
      float x[kMove];
#pragma unroll
      for (int u = 0; u < kMove; ++u) {
        on[u] = compact_entry(a, r, i0 + 256 * u + threadIdx.x, src[u], dst[u]) && src[u] != dst[u];
        x[u] = on[u] ? in[src[u]] : 0.f;
      }
      dma_wait_barrier<0>();
#pragma unroll
      for (int u = 0; u < kMove; ++u)
        if (on[u]) out[dst[u]] = x[u];
    }
    return;
  }
  const int per = 256 / cw, e = threadIdx.x / cw, c = blockIdx.y % columns * cw + threadIdx.x % cw;
  const char* in = a.in[kind] + l * a.il + b * a.ib + h * a.ih + 16 * c;
  char* out = a.out[kind] + l * a.ol + b * a.ob + h * a.oh + 16 * c;
  for (int i0 = 0; i0 < r.n; i0 += per * kMove) {
    u32x4 x[kMove];
#pragma unroll
    for (int u = 0; u < kMove; ++u) {
      on[u] = c < a.nv && compact_entry(a, r, i0 + per * u + e, src[u], dst[u]) && src[u] != dst[u];
      x[u] = on[u] ? *reinterpret_cast<const u32x4*>(in + src[u] * a.is) : u32x4{0, 0, 0, 0};
    }
    dma_wait_barrier<0>();
#pragma unroll
    for (int u = 0; u < kMove; ++u)
      if (on[u]) *reinterpret_cast<u32x4*>(out + dst[u] * a.os) = x[u];
  }
}

}  // namespace
}  // namespace spider

using namespace spider;

extern "C" size_t spider_cache_select_workspace_size(int L, int B, int Hkv, int cap, int shared) {
  return select_shape_ok(L, B, Hkv, cap, shared) ? select_layout((int64_t)L * B * (shared ? 1 : Hkv), cap, shared && Hkv > 1, nullptr,
                                                               nullptr)
                                                 : 0;
}

extern "C" spider_status spider_cache_select(int L, int B, int Hkv, int cap, const float* weights, const int32_t* lens,
                                             int keep, int n_first, int n_last, int shared, int32_t* idx_out,
                                             int32_t* len_out, void* workspace, size_t workspace_bytes,
                                             spider_stream stream) {
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
  SPIDER_REQUIRE((int64_t)L * B * G < (1 << 22) && cap <= (1 << 30), SPIDER_ERR_UNSUPPORTED,
                 "spider_cache_select: layers * samples * head groups below 2^22, cap at most 2^30");
  const size_t need = select_layout((int64_t)L * B * G, cap, G != Hkv, nullptr, nullptr);
  SPIDER_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), SPIDER_ERR_WORKSPACE,
                 "spider_cache_select: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : 0);
  SPIDER_REQUIRE(need == 0 || reinterpret_cast<uintptr_t>(workspace) % 256 == 0, SPIDER_ERR_INVALID_ARG,
                 "spider_cache_select: workspace must be 256-byte aligned");
  // (every row reads lens while one of them writes len_out)
  SPIDER_REQUIRE(len_out + B <= lens || lens + B <= len_out, SPIDER_ERR_INVALID_ARG,
                 "spider_cache_select: len_out must not overlap lens");
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  ProfScope ps(KC_CACHE_SELECT, st);
  const SelectArgs a{weights, lens, idx_out, len_out, L, B, Hkv, G, cap, keep, n_first, n_last};
  if (need) {
    ChunkWs ws;
    select_layout((int64_t)L * B * G, cap, G != Hkv, reinterpret_cast<char*>(workspace), &ws);
    const int chunks = ceil_div(cap, kChunk);
    const unsigned blocks = (unsigned)(L * B * G * chunks);
    cache_select_chunk_kernel<1><<<blocks, kChunkThreads, 0, st>>>(a, ws, chunks);
    cache_select_chunk_kernel<2><<<blocks, kChunkThreads, 0, st>>>(a, ws, chunks);
    cache_select_chunk_kernel<3><<<blocks, kChunkThreads, 0, st>>>(a, ws, chunks);
    cache_select_chunk_kernel<4><<<blocks, kChunkThreads, 0, st>>>(a, ws, chunks);
    SPIDER_LAUNCHED("cache_select_chunk");
    return SPIDER_OK;
  }
  // the smallest block whose registers hold a row
  const unsigned rows = (unsigned)(L * B * G);
  if (cap <= 256 * 16) cache_select_kernel<256, 16><<<rows, 256, 0, st>>>(a);
  else if (cap <= 1024 * 16) cache_select_kernel<1024, 16><<<rows, 1024, 0, st>>>(a);
  else if (cap <= 1024 * 64) cache_select_kernel<1024, 64><<<rows, 1024, 0, st>>>(a);
  else cache_select_kernel<1024, 0><<<rows, 1024, 0, st>>>(a);
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
  const int n_in[4] = {L, B, cap_in, Hkv}, n_out[4] = {L, B, cap_out, Hkv};
  int64_t in[4], out[4];  // bytes; the stride of a dimension of size 1 means nothing
  for (int i = 0; i < 4; ++i) {
    in[i] = n_in[i] == 1 ? 0 : in_strides[i] * es;
    out[i] = n_out[i] == 1 ? 0 : out_strides[i] * es;
    SPIDER_REQUIRE(in[i] >= 0 && out[i] >= 0 && in[i] % 16 == 0 && out[i] % 16 == 0, SPIDER_ERR_INVALID_ARG,
                   "spider_cache_compact: strides must be multiples of 16 bytes");
    SPIDER_REQUIRE(n_out[i] == 1 || out[i] > 0, SPIDER_ERR_INVALID_ARG,
                   "spider_cache_compact: the output's slots must not share memory (a stride of 0)");
    same = same && in[i] == out[i];
  }
  const bool inplace = k_in == k_out;
  SPIDER_REQUIRE(inplace == (v_in == v_out) && (!weights_in || inplace == (weights_in == weights_out)),
                 SPIDER_ERR_INVALID_ARG, "spider_cache_compact: keys, values and weights all move in place or none");
  SPIDER_REQUIRE(!inplace || same, SPIDER_ERR_SHAPE,
                 "spider_cache_compact: in place, the strides and capacities of both sides must be the same");
  SPIDER_REQUIRE((int64_t)L * B * Hkv <= 65535 && n_max <= (1 << 25), SPIDER_ERR_UNSUPPORTED,
                 "spider_cache_compact: L * B * Hkv at most 65535, n_max at most 2^25");
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
  a.il = in[0], a.ib = in[1], a.is = in[2], a.ih = in[3];
  a.ol = out[0], a.ob = out[1], a.os = out[2], a.oh = out[3];
  a.L = L, a.B = B, a.Hkv = Hkv, a.nv = dh * es / 16;
  a.cap_in = cap_in, a.cap_out = cap_out, a.n_max = n_max, a.idx_layers = idx_layers, a.idx_heads = idx_heads;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  ProfScope ps(KC_CACHE_COMPACT, st);
  const unsigned rows = (unsigned)(L * B * Hkv);
  // Columns of 128 bytes, or of 32 where there are few streams to walk.  Measured, columns
  // of 32 / 64 / 128 / 256 bytes: 64 streams of 16384 entries of 256 bytes 350 / 365 / 503 /
  // 863 us; 256 streams of 600, 128 / 256 bytes 27 / 31 us; 1024 streams of 576 136 / 132 us.
  const int cw = (int64_t)L * B * Hkv >= 256 ? 8 : 2;
  if (inplace)
    cache_move_kernel<<<dim3(rows, (unsigned)(ceil_div(a.nv, cw) * (weights_in ? 3 : 2))), 256, 0, st>>>(a, cw);
  else
    cache_copy_kernel<<<dim3((unsigned)ceil_div(n_max, 256 / a.nv), rows), 256, 0, st>>>(a);
  SPIDER_LAUNCHED("cache_compact");
  return SPIDER_OK;
}
