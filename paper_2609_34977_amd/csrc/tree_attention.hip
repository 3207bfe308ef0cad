// Attention of a tree of drafted tokens over a key/value cache
// (spider_tree_attention) and the attention weight every slot receives.
//
//   s(r, j) = scale q_r . k_j,  o_r = sum_j softmax_j(s(r, .)) v_j
// over the slots j that row r = (node t, head h) sees: the context j < lens[b]
// and the nodes u = j - lens[b] whose bit is set in the node's mask.
//
// The rows of a kv head (nodes x heads of its group) read the same keys and values.
// Up to 32 rows a call is bound by those reads (tree_attention_kernel), beyond by
// the softmax and the products (tree_rows_kernel); the splits of the keys meet in
// tree_finish_kernel.  Measured on one MI355X, bf16 of 128, us per call:
//   1 row of 32 kv heads over 200 slots             8.8 (host time; the kernel 8)
//   16 rows of 32 kv heads over 705, weights       15.5
//   4 rows of 16 x 8 kv heads over 32768            352 (6.1 TB/s), with weights 460
//   32 rows of 8 x 8 kv heads over 16384            111..116 (4.7 TB/s)
//   61 / 244 rows of 8 x 8 kv heads over 16384      144 / 244..247
#include <algorithm>
#include <cmath>

#include "attention_tiles.h"
#include "kernels.h"

namespace spider {
namespace {

typedef short short4v __attribute__((ext_vector_type(4)));

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
  float2* stat;     // [B][T][H] (largest score in powers of two, 1 / sum of exponentials), with w_out
  float2* part_ml;  // [B][Hkv][T * G][splits] (largest raw score, sum) of a split
  float* part_o;    // .. [dh] its unscaled output
  float* scores;    // [B][Hkv][tiles][T * G][keys of a tile] raw scores, -inf where not seen, or null
  int64_t qb, qt;         // strides of q, elements
  int64_t kvb, kvs, kvh;  // strides of k and v
  int B, T, H, Hkv, dh, cap;
  float scale;
  int groups, splits, min_tiles;  // of the launch, see TreePlan
  int join_blocks;                // of tree_finish_kernel
};

// The filled slots and live nodes of sample b, clamped to the cache.
__device__ __forceinline__ int2 tree_extent(const TreeArgs& a, int b) {
  const int len = min(max(a.lens[b], 0), a.cap);
  const int nn = a.n_nodes ? min(max(a.n_nodes[b], 0), a.T) : a.T;
  return make_int2(len, min(nn, a.cap - len));
}

// Bits of the KEYS keys from j0 that node t sees: the context, then its mask.
template <int KEYS>
__device__ __forceinline__ uint32_t tree_window(const TreeArgs& a, int b, int t, int j0, int2 ext) {
  const int u0 = j0 - ext.x;  // node of the first key, negative within the context
  uint64_t x;
  if (!a.mask) {
    const int c = t - u0 + 1;
    x = c >= 64 ? ~0ull : (c <= 0 ? 0ull : (1ull << c) - 1ull);
  } else {
    const int W = (a.T + 63) / 64;
    const uint64_t* row = a.mask + ((int64_t)b * a.T + t) * W;
    if (u0 >= 0) {
      const int w = u0 >> 6, sh = u0 & 63;
      x = w < W ? row[w] >> sh : 0ull;
      if (sh && w + 1 < W) x |= row[w + 1] << (64 - sh);
    } else {
      x = u0 <= -64 ? ~0ull : (row[0] << -u0) | ((1ull << -u0) - 1ull);
    }
  }
  const int left = ext.x + ext.y - j0;  // keys up to the last live node
  const uint32_t v = left >= 32 ? ~0u : (1u << max(left, 0)) - 1u;
  return (uint32_t)x & v & (KEYS == 32 ? ~0u : (1u << KEYS) - 1u);
}

// Splits of the keys of one sample and the tiles of each: at most a.splits, each of at
// least a.min_tiles tiles, and no more of them than have a tile (129 tiles in 16 splits of
// 9 are 15): a block without one would end with its first fetches in flight.
struct TreeSplits {
  int n, tiles;
};
__device__ __forceinline__ TreeSplits tree_splits(const TreeArgs& a, int tiles) {
  const int most = max(1, min(a.splits, tiles / a.min_tiles));
  const int per = max(1, (tiles + most - 1) / most);
  return TreeSplits{most == 1 ? 1 : (tiles + per - 1) / per, per};
}

// RT row tiles of a wave: queries, and the running maximum, sum and output of their rows.
template <typename AT, int DH, int RT>
struct RowTiles {
  using T = AttnTile<AT, DH>;
  static constexpr int KEYS = T::KEYS, NS = 4 * T::KT, CPL = T::CPL;  // NS: scores of a lane and row tile
  typename T::Q q[RT];
  int node[RT];
  floatx4 o[RT][CPL];
  float top[RT], sum[RT];
  float p[RT][NS];
  uint32_t seen[RT];  // the lane's keys of the tile that its row sees, bit i for score i
  int bad0 = 0x7fffffff, bad1 = -1;  // the first and last tile with an infinite or NaN value, as far as known

  template <bool FULL>
  __device__ __forceinline__ void start(const TreeArgs& a, int b, int hk, int r0, int R, int lane) {
    const int G = a.H / a.Hkv;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int row = min(r0 + 16 * r + (lane & 15), R - 1);
      node[r] = row / G;
      const AT* qp = reinterpret_cast<const AT*>(a.q) + b * a.qb + node[r] * a.qt + (int64_t)(hk * G + row % G) * a.dh;
      T::template load_q<FULL>(q[r], qp, lane >> 4, a.dh, a.scale < 0.f);
      top[r] = -INFINITY;
      sum[r] = 0.f;
#pragma unroll
      for (int c = 0; c < CPL; ++c) o[r][c] = floatx4{};
    }
  }

  __device__ __forceinline__ void scores(const typename T::K& k) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      floatx4 s[T::KT];
      T::scores(s, k, q[r]);
#pragma unroll
      for (int i = 0; i < NS; ++i) p[r][i] = s[i / 4][i % 4];
    }
  }

  // scores to weights, for the tile of keys from j0; tail: some key is a node, or past the
  // last one; keep (or null): where the tile's scores of the lane's row go (row tile 0)
  template <bool tail>
  __device__ __forceinline__ void soften(const TreeArgs& a, int b, int j0, int2 ext, int g, float sc,
                                         float* keep = nullptr) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      seen[r] = ~0u;
      if constexpr (tail) {
        const uint32_t w = tree_window<KEYS>(a, b, node[r], j0, ext) >> (4 * g);
        seen[r] = (w & 15u) | (T::KT == 2 ? (w >> 12) & 0xF0u : 0u);
#pragma unroll
        for (int i = 0; i < NS; ++i) p[r][i] = (seen[r] >> i) & 1u ? p[r][i] : -INFINITY;
      }
    }
    if (keep) {
#pragma unroll
      for (int i = 0; i < NS; i += 4)
        *reinterpret_cast<floatx4*>(keep + 4 * i + 4 * g) = floatx4{p[0][i], p[0][i + 1], p[0][i + 2], p[0][i + 3]};
    }
    bool grows = false;
    float mx[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      mx[r] = p[r][0];
#pragma unroll
      for (int i = 1; i < NS; ++i) mx[r] = fmaxf(mx[r], p[r][i]);
      float2 x = lanes_x16(mx[r]);
      x = lanes_x32(fmaxf(x.x, x.y));
      mx[r] = fmaxf(x.x, x.y);
      grows = grows || mx[r] * sc > top[r] * sc + kLazyMax || (top[r] == -INFINITY && mx[r] > -INFINITY);
    }
    if (__any(grows)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const float nt = fmaxf(top[r], mx[r]);
        const float f = top[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top[r] - nt) * sc);
        top[r] = nt;
        sum[r] *= f;
#pragma unroll
        for (int c = 0; c < CPL; ++c) o[r][c] *= f;
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const float mc = top[r] == -INFINITY ? 0.f : top[r] * sc;
      float s0 = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        float e = __builtin_amdgcn_exp2f(fmaf(p[r][i], sc, -mc));
        if constexpr (tail) e = (seen[r] >> i) & 1u ? e : 0.f;
        p[r][i] = e;
        s0 += e;
      }
      sum[r] += s0;
    }
  }

  // Infinite and NaN values count for the rows that see them and for no other, but 0 times
  // one of them is NaN.  The values of a tail tile leave the product if they are not finite;
  // those of other tiles, which all rows see, enter it, where they can give NaN for an
  // infinite sum (a weight's low part that is 0 or negative, a weight that has underflowed).
  // settle() puts both right after the loop.

  // whether tile t holds such a value (they become 0)
  template <typename S>
  __device__ __forceinline__ void drop(S& v, int t) {
    const bool dropped = T::drop_nonfinite(v);  // of every tile, whatever the tiles before held
    if (__any(dropped)) {
      bad0 = min(bad0, t);
      bad1 = max(bad1, t);
    }
  }

  // the values of tile t into the outputs
  template <bool tail, typename S>
  __device__ __forceinline__ void add(S& v, int t) {
    if constexpr (tail) drop(v, t);
    T::template values<RT, S>(o, v, p);
  }

  // The outputs, after the tiles t0, t0 + by, .. < full without their nodes and tail tiles
  // behind them: what a row sees of infinite and NaN values is its output.  (If there was
  // one in a full tile, then the output is not finite; the tiles are read again to find it.)
  // channel(c, i): of output o[.][c][i]
  template <bool FULL, typename F>
  __device__ __forceinline__ void settle(const TreeArgs& a, int b, const AT* vb, int t0, int by, int full, int n, int2 ext,
                                         int lane, F&& channel) {
    bool x = false;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) x = x || !(fabsf(o[r][c][i]) < INFINITY);
    if (__any(x)) {
#pragma unroll 1
      for (int t = t0; t < full; t += by) {
        typename T::V v;
        T::template load_v<FULL>(v, vb, a.kvs, t * KEYS, n, lane, a.dh);
        drop(v, t);
      }
    }
    if (bad0 > bad1) return;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int c = 0; c < CPL; ++c) {
        floatx4 s = floatx4{};
#pragma unroll 1
        for (int t = bad0; t <= bad1; t += by)
#pragma unroll 1
          for (int j = t * KEYS; j < min(n, (t + 1) * KEYS); ++j) {
            if (!(tree_window<KEYS>(a, b, node[r], j, ext) & 1u)) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int ch = channel(c, i);
              const float y = ch < a.dh ? T::value(vb + (int64_t)j * a.kvs + ch) : 0.f;
              if (!(fabsf(y) < INFINITY)) s[i] += y;
            }
          }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(fabsf(s[i]) < INFINITY)) o[r][c][i] = s[i];
      }
  }

  // the row's sum, in every lane of its column
  __device__ __forceinline__ float row_sum(int r) const {
    float2 x = lanes_x16(sum[r]);
    x = lanes_x32(x.x + x.y);
    return x.x + x.y;
  }
};

// What a block works on: a unit (sample, kv head, split of its keys) and a group of its
// rows.  The row groups of a unit lie 8 blocks apart: on the same XCD, whose L2 then holds
// the unit's keys and values.
struct TreeWork {
  int b, hk, bh, split, ns, r0, R, n, t0, t1;  // tiles [t0, t1) of the unit's keys
  int2 ext;
};
template <int KEYS, int ROWS>
__device__ __forceinline__ bool tree_work(const TreeArgs& a, TreeWork& w) {
  const int slot = blockIdx.x >> 3;
  const int unit = slot / a.groups * 8 + (blockIdx.x & 7);
  if (unit >= a.B * a.Hkv * a.splits) return false;
  w.split = unit % a.splits;
  w.bh = unit / a.splits;
  w.b = w.bh / a.Hkv;
  w.hk = w.bh % a.Hkv;
  w.ext = tree_extent(a, w.b);
  w.n = w.ext.x + w.ext.y;
  w.R = w.ext.y * (a.H / a.Hkv);
  w.r0 = slot % a.groups * ROWS;
  if (w.r0 >= w.R) return false;
  const int tiles = (w.n + KEYS - 1) / KEYS;
  const TreeSplits s = tree_splits(a, tiles);
  w.ns = s.n;
  if (w.split >= w.ns) return false;
  w.t0 = w.split * s.tiles;
  w.t1 = min(tiles, w.t0 + s.tiles);
  return true;
}

// Few rows: bound by the reads of keys and values, which go straight from memory to the
// registers of the wave that uses them, the next tile's keys on their way during the
// softmax.  4 waves, wave w takes tiles w, w + 4, .. of the block's split; their sums meet
// in LDS.
template <typename AT, int DH, int RT, bool FULL>
__global__ void __launch_bounds__(256, DH* RT <= 128 ? 3 : 1) tree_attention_kernel(TreeArgs a) {
  using Rows = RowTiles<AT, DH, RT>;
  using T = typename Rows::T;
  constexpr int KEYS = T::KEYS, CPL = T::CPL;
  constexpr int ROWS = 16 * RT, LD = DH + 4;
  __shared__ float xm[4][ROWS], xl[4][ROWS];
  __shared__ float xo[4][ROWS][LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m = lane & 15, g = lane >> 4;
  TreeWork w;
  if (!tree_work<KEYS, ROWS>(a, w)) return;
  const int b = w.b, n = w.n, G = a.H / a.Hkv;
  const AT* kb = reinterpret_cast<const AT*>(a.k) + b * a.kvb + w.hk * a.kvh;
  const AT* vb = reinterpret_cast<const AT*>(a.v) + b * a.kvb + w.hk * a.kvh;
  const float sc = fabsf(a.scale) * 1.4426950408889634f;
  Rows rows;
  typename T::K k;
  typename T::V v;
  if (w.t0 + wave < w.t1) T::template load_k<FULL>(k, kb, a.kvs, (w.t0 + wave) * KEYS, n, lane, a.dh);
  rows.template start<FULL>(a, b, w.hk, w.r0, w.R, lane);
  const int64_t tile_scores = (int64_t)a.T * G * KEYS;
  float* kept = RT == 1 && a.scores && m < w.R
                    ? a.scores + (int64_t)w.bh * ((a.cap + KEYS - 1) / KEYS) * tile_scores + m * KEYS : nullptr;
  auto step = [&](int t, auto tail_) {
    constexpr bool tail = decltype(tail_)::value;
    const int j0 = t * KEYS;
    T::template load_v<FULL>(v, vb, a.kvs, j0, n, lane, a.dh);
    rows.scores(k);
    if (t + 4 < w.t1) T::template load_k<FULL>(k, kb, a.kvs, j0 + 4 * KEYS, n, lane, a.dh);
    if constexpr (RT == 1) rows.template soften<tail>(a, b, j0, w.ext, g, sc, kept ? kept + t * tile_scores : nullptr);
    else rows.template soften<tail>(a, b, j0, w.ext, g, sc);
    rows.template add<tail>(v, t);
  };
  int t = w.t0 + wave;
  for (; t < min(w.t1, w.ext.x / KEYS); t += 4) step(t, std::false_type{});
  for (; t < w.t1; t += 4) step(t, std::true_type{});
  rows.template settle<FULL>(a, b, vb, w.t0 + wave, 4, min(w.t1, w.ext.x / KEYS), n, w.ext, lane,
                             [&](int c, int i) { return T::channel(c, 4 * g + i); });

  // the waves' sums onto their common maximum, in wave order
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = rows.row_sum(r);
    if (g == 0) {
      xm[wave][16 * r + m] = rows.top[r];
      xl[wave][16 * r + m] = l;
    }
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) xo[wave][16 * r + m][T::channel(c, 4 * g + i)] = rows.o[r][c][i];
  }
  __syncthreads();
  constexpr int PER = 256 / ROWS >= 4 ? 256 / ROWS : 4;  // threads of a row
  const int c0 = 4 * (tid % PER);
  for (int row = tid / PER; row < min(ROWS, w.R - w.r0); row += 256 / PER) {
    float mx = -INFINITY, l = 0.f, f[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) mx = fmaxf(mx, xm[u][row]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f[u] = xm[u][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((xm[u][row] - mx) * sc);
      // (a row whose scores are all NaN has no maximum, but its sum is NaN and stays)
      l += xm[u][row] == -INFINITY ? xl[u][row] : xl[u][row] * f[u];
    }
    const int rr = w.r0 + row;
    const int64_t out_row = ((int64_t)b * a.T + rr / G) * a.H + w.hk * G + rr % G;
    const int64_t part_row = ((int64_t)w.bh * a.T * G + rr) * a.splits + w.split;
    if (tid % PER == 0) {
      if (w.ns > 1) a.part_ml[part_row] = make_float2(mx, l);
      else if (a.stat) a.stat[out_row] = make_float2(mx == -INFINITY ? 0.f : mx * sc, l == 0.f ? 0.f : 1.f / l);
    }
    for (int c = c0; c < a.dh; c += 4 * PER) {
      floatx4 x = floatx4{};
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += rescaled(xo[u][row][c + i], f[u]);
      if (w.ns > 1) {
        *reinterpret_cast<floatx4*>(a.part_o + part_row * a.dh + c) = x;
      } else {
        attn_store<AT>(a.out, out_row * a.dh + c, x, l);
      }
    }
  }
}

// Many rows (bf16): NW waves of 32 (dh <= 128) or 16 rows each share the keys and values,
// which come through LDS by DMA, two tiles ahead.  244 rows of 128 over 8 x 8 x 16384 keys:
// 247 us, of which 110 the reads alone, the softmax (vector instructions) and the products
// adding to it.  With the weights rounded to bf16 once, a third fewer products and less than
// the other paths keep, it takes 190, and there blocks of 4 waves 187, of 2 281; half of the
// waves half a tile behind the others 209; each row group reading for itself, as with few
// rows, 325.  A tile is 32 rows of DH channels for
// keys and as many for values; 16-byte piece c of key j lies at piece c ^ (j % 16 or less),
// so that both the reads of one piece of 16 keys and those of all pieces of a key spread
// over the banks.
template <int DH, int NW, bool FULL>
__global__ void __launch_bounds__(64 * NW, 2) tree_rows_kernel(TreeArgs a) {
  constexpr int RT = DH == 256 ? 1 : 2;
  using Rows = RowTiles<uint16_t, DH, RT>;
  using T = typename Rows::T;
  constexpr int CPL = T::CPL, ROWS = 16 * RT * NW;
  constexpr int PIECES = DH / 8, SWZ = PIECES < 16 ? PIECES - 1 : 15;  // 16-byte pieces of a row
  constexpr int TILE = 32 * DH, STAGES = 3;                             // elements of a key or value tile
  __shared__ __align__(16) uint16_t buf[STAGES][2][TILE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, g = lane >> 4;
  TreeWork w;
  if (!tree_work<32, ROWS>(a, w)) return;
  const int b = w.b, n = w.n, G = a.H / a.Hkv;
  const uint16_t* kb = reinterpret_cast<const uint16_t*>(a.k) + b * a.kvb + w.hk * a.kvh;
  const uint16_t* vb = reinterpret_cast<const uint16_t*>(a.v) + b * a.kvb + w.hk * a.kvh;
  const float sc = fabsf(a.scale) * 1.4426950408889634f;
  const uint32_t lds0 = lds_offset(&buf[0][0][0]);
  // A DMA of a wave fills 1 KB, 64 / PIECES rows.  Every wave fetches the same rows of keys
  // and values, KD pieces of each (width 64 in 8 waves: one piece, of keys or of values).
  constexpr int KD = DH / 16 / NW, DMAS = KD ? 2 * KD : 1;
  const int last_piece = a.dh / 8 - 1;
  auto fetch = [&](int t) {
    const uint32_t to = lds0 + (uint32_t)((t - w.t0) % STAGES * 4 * TILE);
    if constexpr (KD > 0) {
#pragma unroll
      for (int i = 0; i < KD; ++i) {
        const int part = i * NW + wave, j = part * (64 / PIECES) + lane / PIECES, c = (lane % PIECES) ^ (j & SWZ);
        const int64_t off = (int64_t)min(32 * t + j, n - 1) * a.kvs + 8 * (FULL ? c : min(c, last_piece));
        dma16(kb + off, to + part * 1024);
        dma16(vb + off, to + 2 * TILE + part * 1024);
      }
    } else {
      const int part = wave % (NW / 2), j = part * (64 / PIECES) + lane / PIECES, c = (lane % PIECES) ^ (j & SWZ);
      const int64_t off = (int64_t)min(32 * t + j, n - 1) * a.kvs + 8 * (FULL ? c : min(c, last_piece));
      dma16((wave < NW / 2 ? kb : vb) + off, to + (wave < NW / 2 ? 0 : 2 * TILE) + part * 1024);
    }
  };
  Rows rows;
  rows.template start<FULL>(a, b, w.hk, w.r0 + 16 * RT * wave, w.R, lane);
  dma_wait_all();  // the queries are here: from now on only the DMAs count as loads in flight
  fetch(w.t0);
  if (w.t0 + 1 < w.t1) fetch(w.t0 + 1);
  auto step = [&](int t, auto tail_) {
    constexpr bool tail = decltype(tail_)::value;
    // tile t has landed, and every wave is done with tile t - 1, whose place tile t + 2 takes
    if (t + 1 < w.t1) dma_wait_barrier<DMAS>();
    else dma_wait_barrier<0>();
    if (t + 2 < w.t1) fetch(t + 2);
    const uint16_t* ks = buf[(t - w.t0) % STAGES][0];
    const uint16_t* vs = buf[(t - w.t0) % STAGES][1];
    typename T::K k;
#pragma unroll
    for (int u = 0; u < T::KT; ++u)
#pragma unroll
      for (int i = 0; i < T::NK; ++i) {
        const int c = 4 * i + g;
        u32x4 x = *reinterpret_cast<const u32x4*>(ks + (16 * u + m) * DH + 8 * (c ^ (m & SWZ)));
        if (!FULL && c > last_piece) x = u32x4{0, 0, 0, 0};
        k.f[u][i] = __builtin_bit_cast(bf16x8, x);
      }
    rows.scores(k);
    // the value operands by transposing reads: 16 lanes read four keys of 16 channels, a lane
    // gets the four keys of channel 16 n + lane % 16
    typename T::Ops v;
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
      u32x4 x;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = 16 * e + 4 * g + m / 4, piece = 2 * c + m % 4 / 2;
        const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) short4v*)(vs + j * DH + 8 * (piece ^ (j & SWZ)) + 4 * (m % 2)));
        const uint2 z = __builtin_bit_cast(uint2, y);
        x[2 * e] = z.x;
        x[2 * e + 1] = z.y;
      }
      v.f[c] = x;
    }
    rows.template soften<tail>(a, b, 32 * t, w.ext, g, sc);
    rows.template add<tail>(v, t);
  };
  int t = w.t0;
  for (; t < min(w.t1, w.ext.x / 32); ++t) step(t, std::false_type{});
  for (; t < w.t1; ++t) step(t, std::true_type{});
  rows.template settle<FULL>(a, b, vb, w.t0, 1, min(w.t1, w.ext.x / 32), n, w.ext, lane,
                             [&](int c, int i) { return 16 * c + 4 * g + i; });

#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = rows.row_sum(r), top = rows.top[r];
    const int rr = w.r0 + 16 * (RT * wave + r) + m;
    if (rr >= w.R) continue;
    const int64_t out_row = ((int64_t)b * a.T + rr / G) * a.H + w.hk * G + rr % G;
    const int64_t part_row = ((int64_t)w.bh * a.T * G + rr) * a.splits + w.split;
    if (g == 0) {
      if (w.ns > 1) a.part_ml[part_row] = make_float2(top, l);
      else if (a.stat) a.stat[out_row] = make_float2(top == -INFINITY ? 0.f : top * sc, l == 0.f ? 0.f : 1.f / l);
    }
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
      const int ch = 16 * c + 4 * g;  // of four consecutive outputs
      if (!FULL && ch >= a.dh) continue;
      if (w.ns > 1) *reinterpret_cast<floatx4*>(a.part_o + part_row * a.dh + ch) = rows.o[r][c];
      else attn_store<uint16_t>(a.out, out_row * a.dh + ch, rows.o[r][c], l);
    }
  }
}

// One launch after the attention: blocks below a.join_blocks join the splits of the rows (a
// wave per row with few splits, else a block), the others add up the weights from the kept
// scores.
// Neither waits for the other: a weights block joins its rows' statistics itself.
// Join: groups of dh / 4 threads, a thread per four channels, take every ng-th split, their
// sums meet in LDS in group order.  Weights: a thread per four slots, all live rows of the
// head group in order.
constexpr int kWaveJoin = 8;  // splits that a wave joins
template <typename AT, int THREADS>
__device__ __forceinline__ void tree_join(const TreeArgs& a, float sc) {
  __shared__ float red[4];
  __shared__ floatx4 xs_[256];
  __shared__ float ls_[256];
  constexpr int TEAMS = 256 / THREADS;
  const int team = threadIdx.x / THREADS, tid = threadIdx.x % THREADS;
  floatx4* xs = xs_ + team * THREADS;
  float* ls = ls_ + team * THREADS;
  auto sync = [] {
    if constexpr (THREADS == 64) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    else __syncthreads();
  };
  const int r = blockIdx.x * TEAMS + team, h = r % a.H, t = r / a.H % a.T, b = r / a.H / a.T;
  if (b >= a.B) return;
  const int2 ext = tree_extent(a, b);
  if (t >= ext.y) return;
  constexpr int KEYS = AttnTile<AT, 64>::KEYS;
  const int ns = tree_splits(a, (ext.x + ext.y + KEYS - 1) / KEYS).n;
  if (ns == 1) return;
  const int G = a.H / a.Hkv, hk = h / G;
  const int64_t part = (((int64_t)b * a.Hkv + hk) * a.T * G + (int64_t)t * G + h % G) * a.splits;
  float mx = -INFINITY;
  for (int s = tid; s < ns; s += THREADS) mx = fmaxf(mx, a.part_ml[part + s].x);
  mx = wave_max(mx);
  if constexpr (THREADS == 256) {
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  }
  const int per = a.dh / 4, ng = THREADS / per, grp = tid / per, c = 4 * (tid % per);
  float l = 0.f;
  floatx4 x = floatx4{};
  if (grp < ng) {
    for (int s0 = grp; s0 < ns; s0 += 4 * ng) {
      float2 ml[4];
      floatx4 o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int s = min(s0 + u * ng, ns - 1);
        ml[u] = a.part_ml[part + s];
        o[u] = *reinterpret_cast<const floatx4*>(a.part_o + (part + s) * a.dh + c);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (s0 + u * ng >= ns) break;
        const float f = ml[u].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[u].x - mx) * sc);
        // (a row whose scores are all NaN has no maximum, but its sum is NaN and stays)
        l += ml[u].x == -INFINITY ? ml[u].y : ml[u].y * f;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += rescaled(o[u][i], f);
      }
    }
  }
  xs[tid] = x;
  ls[tid] = l;
  sync();
  if (grp > 0) return;
  for (int i = 1; i < ng; ++i) {
    x += xs[i * per + tid];
    l += ls[i * per + tid];
  }
  const int64_t row = ((int64_t)b * a.T + t) * a.H + h;
  attn_store<AT>(a.out, row * a.dh + c, x, l);
  if (a.stat && tid == 0) a.stat[row] = make_float2(mx == -INFINITY ? 0.f : mx * sc, l == 0.f ? 0.f : 1.f / l);
}

template <typename AT>
__global__ void __launch_bounds__(256) tree_finish_kernel(TreeArgs a) {
  constexpr int KEYS = AttnTile<AT, 64>::KEYS;
  __shared__ float2 st[16];
  const float sc = fabsf(a.scale) * 1.4426950408889634f;
  if ((int)blockIdx.x < a.join_blocks) {
    if (a.splits <= kWaveJoin) tree_join<AT, 64>(a, sc);
    else tree_join<AT, 256>(a, sc);
    return;
  }
  const int blk = blockIdx.x - a.join_blocks, tid = threadIdx.x;
  const int blocks = (a.cap + 1023) / 1024, bh = blk / blocks, b = bh / a.Hkv, hk = bh % a.Hkv;
  const int G = a.H / a.Hkv;
  const int2 ext = tree_extent(a, b);
  const int n = ext.x + ext.y, R = ext.y * G;
  const int j = (blk % blocks * 256 + tid) * 4;
  if (blk % blocks * 1024 >= n) return;
  // (the first rows' scores on their way before their statistics)
  const float* s = a.scores + ((int64_t)bh * ((a.cap + KEYS - 1) / KEYS) + j / KEYS) * a.T * G * KEYS + j % KEYS;
  floatx4 x[8];
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (j < n && u < R) x[u] = *reinterpret_cast<const floatx4*>(s + u * KEYS);
  const int ns = tree_splits(a, (n + KEYS - 1) / KEYS).n;
  if (ns == 1) {
    if (tid < R) st[tid] = a.stat[((int64_t)b * a.T + tid / G) * a.H + hk * G + tid % G];
  } else {
    // 16 lanes per row, every 16th split each
    const int r = tid / 16, k = tid % 16;
    const float2* ml = a.part_ml + ((int64_t)bh * a.T * G + max(0, min(r, R - 1))) * a.splits;
    float mx = -INFINITY, l = 0.f;
    for (int i = k; i < ns; i += 16) mx = fmaxf(mx, ml[i].x);
    mx = fmaxf(mx, lane_dpp<kDppRor8>(mx));
    mx = fmaxf(mx, lane_dpp<kDppRor4>(mx));
    mx = fmaxf(mx, lane_dpp<kDppX2>(mx));
    mx = fmaxf(mx, lane_dpp<kDppX1>(mx));
    for (int i = k; i < ns; i += 16) {
      const float2 v = ml[i];
      l += v.x == -INFINITY ? v.y : v.y * __builtin_amdgcn_exp2f((v.x - mx) * sc);
    }
    l = row16_sum(l);
    if (k == 0) st[r] = make_float2(mx == -INFINITY ? 0.f : mx * sc, l == 0.f ? 0.f : 1.f / l);
  }
  __syncthreads();
  if (j >= n) return;
  floatx4 sum = floatx4{};
  for (int r0 = 0; r0 < R; r0 += 8) {
    if (r0 > 0) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r0 + u < R) x[u] = *reinterpret_cast<const floatx4*>(s + (r0 + u) * KEYS);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (r0 + u >= R) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(x[u][i], sc, -st[r0 + u].x)) * st[r0 + u].y;
        sum[i] += x[u][i] == -INFINITY ? 0.f : e;
      }
    }
  }
  const int64_t at = (int64_t)bh * a.cap + j;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (j + i < n) a.w_out[at + i] = (j + i < ext.x && a.w_in ? a.w_in[at + i] : 0.f) + sum[i];
}

// The weight of every slot, of more rows than keep their scores: a wave per NT tiles of keys
// of one kv head, which stay in registers, all live rows of the head group in tiles of 16;
// exp2(s - max) / sum from the rows' final statistics.  Two tiles share each reading of the
// queries (244 rows over 8 x 8 x 16384 keys, whole call with the attention at 190 us: 438 ->
// 355, and 407 with the attention at 247), where that
// leaves enough blocks (70 rows over 2 x 8 x 500 keys, whole call: one tile 29.5, two 33.4)
// and registers (width 256 has none).
template <typename AT, int DH, bool FULL, int NT>
__global__ void __launch_bounds__(256) tree_weights_kernel(TreeArgs a) {
  using T = AttnTile<AT, DH>;
  constexpr int KEYS = T::KEYS, NS = 4 * T::KT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m = lane & 15, g = lane >> 4;
  const int blocks = (a.cap + 4 * NT * KEYS - 1) / (4 * NT * KEYS), bh = blockIdx.x / blocks;
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const int G = a.H / a.Hkv;
  const int2 ext = tree_extent(a, b);
  const int n = ext.x + ext.y, R = ext.y * G;
  const int j0 = (4 * (blockIdx.x % blocks) + wave) * NT * KEYS;
  if (j0 >= n) return;
  const float sc = fabsf(a.scale) * 1.4426950408889634f;
  typename T::K k[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u)
    T::template load_k<FULL>(k[u], reinterpret_cast<const AT*>(a.k) + b * a.kvb + hk * a.kvh, a.kvs, j0 + u * KEYS, n,
                             lane, a.dh);
  const bool tail = j0 + NT * KEYS > ext.x;
  float acc[NT][NS] = {};
  const int dt = 16 / G, dg = 16 % G;
  int t = m / G, gi = m % G;  // node and head of the group of row r0 + m
  for (int r0 = 0; r0 < R; r0 += 16) {
    const bool on = r0 + m < R;
    const int node = on ? t : ext.y - 1, h = hk * G + (on ? gi : G - 1);
    typename T::Q q;
    T::template load_q<FULL>(q, reinterpret_cast<const AT*>(a.q) + b * a.qb + node * a.qt + (int64_t)h * a.dh, g, a.dh,
                             a.scale < 0.f);
    const float2 st = a.stat[((int64_t)b * a.T + node) * a.H + h];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      floatx4 s[T::KT];
      T::scores(s, k[u], q);
      if (tail || r0 + 16 > R) {
        const uint32_t w = (on ? tree_window<KEYS>(a, b, node, j0 + u * KEYS, ext) : 0u) >> (4 * g);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], sc, -st.x)) * st.y;
          acc[u][i] += (w >> (i / 4 * 16 + i % 4)) & 1u ? e : 0.f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < NS; ++i)
          acc[u][i] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], sc, -st.x)), st.y, acc[u][i]);
      }
    }
    t += dt;
    gi += dg;
    if (gi >= G) {
      gi -= G;
      ++t;
    }
  }
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const float x = row16_sum(acc[u][i]);
      const int j = j0 + u * KEYS + 16 * (i / 4) + 4 * g + i % 4;
      const int64_t at = (int64_t)bh * a.cap + j;
      if (m == i && j < n) a.w_out[at] = (j < ext.x && a.w_in ? a.w_in[at] : 0.f) + x;
    }
}

// Tiles, row groups and splits of a call, and its workspace.
struct TreePlan {
  int dhp;     // kernel width: 64, 128 or 256
  int rt;      // row tiles of a wave of tree_attention_kernel, or 0:
  int nw;      // waves of tree_rows_kernel
  int groups;  // row groups of a unit
  int splits, min_tiles;
  bool kept;  // the weights come from kept scores
  size_t ml_off, o_off, score_off, bytes;
};

TreePlan tree_plan(int B, int T, int H, int Hkv, int dh, int cap, spider_dtype dtype, bool weights) {
  TreePlan p{};
  const bool bf16 = dtype == SPIDER_BF16;
  const int R = T * (H / Hkv), keys = bf16 ? 32 : 16;
  p.dhp = dh <= 64 ? 64 : (dh <= 128 ? 128 : 256);
  const int wave_rows = p.dhp == 256 ? 16 : 32;
  int rows, target;
  if (!bf16 || R <= wave_rows) {
    p.rt = R <= 16 ? 1 : 2;
    rows = 16 * p.rt;
    target = 768;
  } else {
    // (width 256 has no registers for two waves per SIMD)
    p.nw = R <= 2 * wave_rows ? 2 : (R <= 4 * wave_rows || p.dhp == 256 ? 4 : 8);
    rows = wave_rows * p.nw;
    // eight waves per CU; width 256 leaves LDS for one block
    target = p.dhp == 256 ? 256 : 256 * 8 / p.nw;
  }
  p.groups = ceil_div(R, rows);
  // At least eight tiles per split.  Measured with 4 / 8 / 16, us on the device: 16 rows of
  // 32 heads over 705 slots with weights 13.6 / 15.1 / 17.8; 32 rows of 8 heads over 2000
  // 10.6 / 12.9 / 15.3; 4 x 1 row of 32 heads over 705 16.4 / 16.1 / 14.2; 244 rows of 8
  // heads over 2000 29.1 / 29.4 / 37.9; fp32, 2 x 13 rows of 8 heads over 1500 with weights
  // 13.8 / 12.8 / 14.6; 4 rows of 8 heads over 20000 24.0 / 24.0 / 24.9.  (Four would gain on
  // short bf16 caches with idle CUs and lose in fp32.)
  p.min_tiles = 8;
  const int64_t units = (int64_t)B * Hkv * p.groups;
  const int tiles = ceil_div(cap, keys);
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>((target + units - 1) / units, tiles / p.min_tiles));
  size_t off = weights ? align_up((size_t)B * T * H * sizeof(float2), 256) : 0;
  p.ml_off = off;
  if (p.splits > 1) {
    const size_t rows_ = (size_t)B * T * H * p.splits;
    off = align_up(off + rows_ * sizeof(float2), 256);
    p.o_off = off;
    off = align_up(off + rows_ * dh * sizeof(float), 256);
  }
  // The weights of up to 16 rows come from the scores, kept in fp32 (8 bytes a row and key,
  // written and read), those of more rows from a second pass over the keys (2 dh bytes a
  // key, and the products again).  Measured, 4 rows of 128 over 16 x 8 x 32768 keys: 468 us
  // with kept scores, 605 us with the second pass (352 us without weights).
  p.score_off = off;
  if (weights && p.rt == 1) {
    p.kept = true;
    off = align_up(off + (size_t)B * Hkv * R * tiles * keys * sizeof(float), 256);
  }
  p.bytes = off;
  return p;
}

unsigned tree_blocks(const TreeArgs& a) { return (unsigned)((a.B * a.Hkv * a.splits + 7) / 8 * 8 * a.groups); }

template <typename AT, int DH, int RT>
void launch_tree(const TreeArgs& a, hipStream_t st) {
  if (a.dh == DH) tree_attention_kernel<AT, DH, RT, true><<<tree_blocks(a), 256, 0, st>>>(a);
  else tree_attention_kernel<AT, DH, RT, false><<<tree_blocks(a), 256, 0, st>>>(a);
}

template <int DH, int NW>
void launch_tree_rows(const TreeArgs& a, hipStream_t st) {
  if (a.dh == DH) tree_rows_kernel<DH, NW, true><<<tree_blocks(a), 64 * NW, 0, st>>>(a);
  else tree_rows_kernel<DH, NW, false><<<tree_blocks(a), 64 * NW, 0, st>>>(a);
}

template <typename AT, int DH, int NT>
void launch_tree_weights(const TreeArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)ceil_div(a.cap, 4 * NT * AttnTile<AT, DH>::KEYS) * (unsigned)(a.B * a.Hkv);
  if (a.dh == DH) tree_weights_kernel<AT, DH, true, NT><<<grid, 256, 0, st>>>(a);
  else tree_weights_kernel<AT, DH, false, NT><<<grid, 256, 0, st>>>(a);
}

template <typename AT, int DH>
spider_status run_tree(const TreeArgs& a, const TreePlan& p, hipStream_t st) {
  {
    ProfScope ps(KC_TREE_ATTN, st);
    if (p.rt == 1) launch_tree<AT, DH, 1>(a, st);
    else if constexpr (sizeof(AT) == 4) launch_tree<AT, DH, 2>(a, st);
    else if (p.nw == 2) launch_tree_rows<DH, 2>(a, st);
    else if (p.nw == 4) launch_tree_rows<DH, 4>(a, st);
    else if constexpr (DH <= 128) {
      if (p.nw == 8) launch_tree_rows<DH, 8>(a, st);
      else launch_tree<AT, DH, 2>(a, st);
    }
    SPIDER_LAUNCHED("tree_attention");
  }
  const unsigned weight_blocks = a.scores ? (unsigned)ceil_div(a.cap, 1024) * (unsigned)(a.B * a.Hkv) : 0u;
  if (a.join_blocks + weight_blocks > 0) {
    ProfScope ps(a.scores ? KC_TREE_WEIGHTS : KC_TREE_ATTN, st);
    tree_finish_kernel<AT><<<a.join_blocks + weight_blocks, 256, 0, st>>>(a);
    SPIDER_LAUNCHED("tree_finish");
  }
  if (a.w_out && !a.scores) {
    ProfScope ps(KC_TREE_WEIGHTS, st);
    const bool two = (int64_t)a.B * a.Hkv * ceil_div(a.cap, 8 * AttnTile<AT, DH>::KEYS) >= 512;
    if constexpr (DH <= 128) {
      if (two) launch_tree_weights<AT, DH, 2>(a, st);
      else launch_tree_weights<AT, DH, 1>(a, st);
    } else {
      launch_tree_weights<AT, DH, 1>(a, st);
    }
    SPIDER_LAUNCHED("tree_weights");
  }
  return SPIDER_OK;
}

template <typename AT>
spider_status run_tree(const TreeArgs& a, const TreePlan& p, hipStream_t st) {
  return p.dhp == 64 ? run_tree<AT, 64>(a, p, st) : (p.dhp == 128 ? run_tree<AT, 128>(a, p, st) : run_tree<AT, 256>(a, p, st));
}

bool tree_shape_ok(int B, int T, int H, int Hkv, int dh, int cap, spider_dtype dtype) {
  return B >= 1 && B <= 65535 && T >= 1 && T <= kTreeMaxNodes && H >= 1 && H <= 65535 && Hkv >= 1 && H % Hkv == 0 &&
         dh >= 1 && dh <= kTreeMaxDh && cap >= 1 && (int64_t)B * H * T < (1 << 24) &&
         (int64_t)B * Hkv * ceil_div(cap, 64) < (1 << 24) && (dtype == SPIDER_BF16 || dtype == SPIDER_F32);
}

}  // namespace
}  // namespace spider

using namespace spider;

extern "C" size_t spider_tree_attention_workspace_size(int B, int T, int H, int Hkv, int dh, int cap,
                                                       spider_dtype dtype, int weights) {
  if (!tree_shape_ok(B, T, H, Hkv, dh, cap, dtype)) return 0;
  return tree_plan(B, T, H, Hkv, dh, cap, dtype, weights != 0).bytes;
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
  // blocks of the largest launch (a grid holds 2^24 blocks of 256 threads)
  SPIDER_REQUIRE((int64_t)B * H * T < (1 << 24) && (int64_t)B * Hkv * ceil_div(cap, 64) < (1 << 24),
                 SPIDER_ERR_UNSUPPORTED, "spider_tree_attention: B * H * T or B * Hkv * cap / 64 reach 2^24");
  // the stride of a dimension of size 1 means nothing
  if (B == 1) q_stride_b = kv_stride_b = 0;
  if (T == 1) q_stride_t = 0;
  if (cap == 1) kv_stride_s = 0;
  if (Hkv == 1) kv_stride_h = 0;
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
  const TreePlan p = tree_plan(B, T, H, Hkv, dh, cap, dtype, weights_out != nullptr);
  const size_t need = p.bytes;
  SPIDER_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), SPIDER_ERR_WORKSPACE,
                 "spider_tree_attention: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : 0);
  SPIDER_REQUIRE(need == 0 || reinterpret_cast<uintptr_t>(workspace) % 256 == 0, SPIDER_ERR_INVALID_ARG,
                 "spider_tree_attention: workspace must be 256-byte aligned");
  char* ws = reinterpret_cast<char*>(workspace);
  TreeArgs a{q, k, v, out, lens, n_nodes, tree_mask, weights_in, weights_out, nullptr, nullptr, nullptr,
             nullptr, q_stride_b, q_stride_t, kv_stride_b, kv_stride_s, kv_stride_h, B, T, H, Hkv, dh, cap, scale,
             p.groups, p.splits, p.min_tiles,
             p.splits == 1 ? 0 : (p.splits <= kWaveJoin ? ceil_div(B * T * H, 4) : B * T * H)};
  if (weights_out) a.stat = reinterpret_cast<float2*>(ws);
  if (p.splits > 1) {
    a.part_ml = reinterpret_cast<float2*>(ws + p.ml_off);
    a.part_o = reinterpret_cast<float*>(ws + p.o_off);
  }
  if (p.kept) a.scores = reinterpret_cast<float*>(ws + p.score_off);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  return dtype == SPIDER_BF16 ? run_tree<uint16_t>(a, p, st) : run_tree<float>(a, p, st);
}
