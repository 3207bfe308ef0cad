// Attention of a chunk of new tokens per sequence over a paged cache (spider_paged_attention).
//
//   s(r, j) = scale q_r . k_j,  o_r = sum_j softmax_j(s(r, .)) v_j
// over the slots j that row r = (new token, head) sees: those up to its own position, within the
// window, whose page is present.
//
// The rows of a kv head (tokens x heads of its group) read the same keys and values.  Few rows are
// bound by those reads (paged_few_kernel), many by the softmax and the products
// (paged_chunk_kernel); splits of the keys meet in paged_join_kernel.  The softmax numerators
// enter the product with v in v's type, rounded once, and their sum is that of the rounded ones:
// in bf16 an output is then about 1.3 times as far from the exact one as its own rounding makes it.
#include <algorithm>
#include <cmath>

#include "attention_tiles.h"
#include "kernels.h"
#include "paged.h"

namespace spider {
namespace {

typedef short short4v __attribute__((ext_vector_type(4)));

struct ChunkArgs {
  PagedArgs p;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float2* part_ml;  // [N * H][splits] (largest raw score, sum) of a split
  float* part_o;    // .. [dh] its unscaled output
  int64_t qs;
  int H, Hkv, dh, window;
  float scale;
  int row_blocks, splits, min_tiles;
};

// What a block works on: rows r0 .. of the R rows of a sequence and kv head, tiles [t0, t1) of
// its keys, which are split `split` of ns.
struct ChunkWork {
  PagedSeq s;
  int b, hk, split, ns, r0, R, t0, t1;
};

// The tiles that any of the rows r0 .. r0 + rows - 1 sees, and their splits: at most a.splits, each
// of at least a.min_tiles tiles, and no more of them than have a tile.
__device__ __forceinline__ void chunk_tiles(const ChunkArgs& a, ChunkWork& w, int keys, int rows) {
  const int G = a.H / a.Hkv, first = w.s.len - w.s.rows + w.r0 / G;
  const int last = w.s.len - w.s.rows + (min(w.r0 + rows, w.R) - 1) / G;
  const int lo = a.window > 0 ? max(0, first - a.window + 1) : 0;
  w.t0 = last < 0 ? 0 : lo / keys;
  const int end = last < 0 ? 0 : last / keys + 1, n = end - w.t0;
  const int most = max(1, min(a.splits, n / a.min_tiles));
  const int per = max(1, (n + most - 1) / most);
  w.ns = most == 1 ? 1 : (n + per - 1) / per;
  w.t0 += w.split * per;
  w.t1 = w.ns == 1 ? end : min(end, w.t0 + per);
}

// Row blocks of ROWS rows: those of sequence b start at number floor(cu[b] G / ROWS) + b, which
// leaves every sequence as many as it needs, so that nobody has to count them beforehand; the
// later rows of a sequence, which see more, come first.  Blocks of a (kv head, split) lie on one
// XCD, whose L2 then holds its keys and values, where their number is a multiple of the 8 XCDs.
template <int KEYS, int ROWS>
__device__ __forceinline__ bool chunk_work(const ChunkArgs& a, ChunkWork& w) {
  const int units = a.Hkv * a.splits, G = a.H / a.Hkv;
  int unit, rb;
  if (units % 8 == 0) {
    const int slot = blockIdx.x >> 3;
    unit = slot / a.row_blocks * 8 + (blockIdx.x & 7);
    rb = slot % a.row_blocks;
  } else {
    unit = blockIdx.x % units;
    rb = blockIdx.x / units;
  }
  w.hk = unit % a.Hkv;
  w.split = unit / a.Hkv;
  auto at = [&](int b) { return (int)((int64_t)paged_start(a.p, b) * G / ROWS) + b; };
  w.b = last_at_most(a.p.B, rb, at);
  if (w.b < 0) return false;
  w.s = paged_seq(a.p, w.b);
  w.R = w.s.rows * G;
  const int i = (w.R + ROWS - 1) / ROWS - 1 - (rb - at(w.b));
  if (i < 0) return false;
  w.r0 = i * ROWS;
  chunk_tiles(a, w, KEYS, ROWS);
  return w.split < w.ns;
}

// The table entries of a sequence, 64 at a time in the lanes of a wave.
struct PageIds {
  const int32_t* row;
  int last, n_pages, base, id;
  __device__ __forceinline__ void start(const ChunkArgs& a, const ChunkWork& w) {
    row = a.p.table + w.b * a.p.table_stride;
    last = (w.s.len - 1) >> a.p.shift;
    n_pages = a.p.n_pages;
    base = -64;
  }
  // entry i, the same in every lane and not below earlier ones; -1: absent
  __device__ __forceinline__ int get(int i) {
    if (i >= base + 64) {
      base = i;
      const int at = i + (int)(threadIdx.x & 63);
      id = at <= last ? row[at] : -1;
      id = (uint32_t)id < (uint32_t)n_pages ? id : -1;
    }
    return __builtin_amdgcn_readlane(id, i - base);
  }
};

// Where the keys of a tile lie: element offsets of its groups of eight, and which of its keys
// there are (bits).  An absent page's keys are read from page 0 and not seen.
template <int KEYS>
struct TileAt {
  int64_t off[KEYS / 8];
  uint32_t present;
  __device__ __forceinline__ void find(const ChunkArgs& a, PageIds& ids, int j0) {
    present = 0;
#pragma unroll
    for (int u = 0; u < KEYS / 8; ++u) {
      const int j = j0 + 8 * u, id = ids.get(j >> a.p.shift);
      present |= id >= 0 ? 0xFFu << (8 * u) : 0u;
      off[u] = max(id, 0) * a.p.sp + (j & ((1 << a.p.shift) - 1)) * a.p.ss;
    }
  }
};

// Bits of the keys from j0 that a row at position pos sees, of those that are present.
__device__ __forceinline__ uint32_t chunk_window(uint32_t present, int pos, int window, int j0) {
  const int c = pos - j0 + 1;
  uint32_t x = c >= 32 ? ~0u : (1u << max(c, 0)) - 1u;
  if (window > 0) {
    const int d = c - window;  // keys before the window
    x &= d >= 32 ? 0u : ~0u << max(d, 0);
  }
  return x & present;
}

// RT row tiles of a wave: queries, and the running maximum, sum and output of their rows.
template <typename AT, int DH, int RT>
struct ChunkRows {
  using T = AttnTile<AT, DH>;
  static constexpr int KEYS = T::KEYS, NS = 4 * T::KT, CPL = T::CPL;
  static constexpr bool BF16 = sizeof(AT) == 2;
  typename T::Q q[RT];
  int pos[RT];
  int first, last;  // positions of the wave's rows
  floatx4 o[RT][CPL];
  floatx4 sum[RT];  // bf16: the same sum four times (a product with ones); fp32: element 0, of the lane's keys
  float top[RT];
  float p[RT][NS];
  int bad0 = 0x7fffffff, bad1 = -1;  // the first and last masked tile with an infinite or NaN value

  template <bool FULL>
  __device__ __forceinline__ void start(const ChunkArgs& a, const ChunkWork& w, int r0, int lane) {
    const int G = a.H / a.Hkv, p0 = w.s.len - w.s.rows;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int row = min(r0 + 16 * r + (lane & 15), w.R - 1), t = row / G;
      pos[r] = p0 + t;
      const AT* qp = reinterpret_cast<const AT*>(a.q) + (int64_t)(w.s.start + t) * a.qs + (int64_t)(w.hk * G + row % G) * a.dh;
      T::template load_q<FULL>(q[r], qp, lane >> 4, a.dh, a.scale < 0.f);
      top[r] = -INFINITY;
      sum[r] = floatx4{};
#pragma unroll
      for (int c = 0; c < CPL; ++c) o[r][c] = floatx4{};
    }
    first = p0 + min(r0, w.R - 1) / G;
    last = p0 + min(r0 + 16 * RT - 1, w.R - 1) / G;
  }

  // whether some row of the wave does not see some key of the tile from j0
  __device__ __forceinline__ bool masked(uint32_t present, int window, int j0) const {
    return present != (KEYS == 32 ? ~0u : 0xFFFFu) || j0 + KEYS - 1 > first || (window > 0 && j0 <= last - window);
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

  // scores to weights
  __device__ __forceinline__ void soften(uint32_t present, int window, int j0, bool mask, int g, float sc) {
    uint32_t seen[RT];
    if (mask) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint32_t x = chunk_window(present, pos[r], window, j0) >> (4 * g);
        seen[r] = (x & 15u) | (T::KT == 2 ? (x >> 12) & 0xF0u : 0u);
#pragma unroll
        for (int i = 0; i < NS; ++i) p[r][i] = (seen[r] >> i) & 1u ? p[r][i] : -INFINITY;
      }
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
#pragma unroll
      for (int i = 0; i < NS; ++i) p[r][i] = __builtin_amdgcn_exp2f(fmaf(p[r][i], sc, -mc));
    }
    if (mask) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < NS; ++i) p[r][i] = (seen[r] >> i) & 1u ? p[r][i] : 0.f;
    }
  }

  // the values of tile t into the outputs.  Infinite and NaN values of a masked tile must not
  // reach the rows that do not see them (0 times one of them is NaN): they leave the product, and
  // settle() puts them right after the loop.
  template <typename S>
  __device__ __forceinline__ void add(S& v, bool mask, int t) {
    if (mask) {
      const bool dropped = T::drop_nonfinite(v);
      if (__any(dropped)) {
        bad0 = min(bad0, t);
        bad1 = max(bad1, t);
      }
    }
    if constexpr (BF16) {
      const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
      bf16x8 w[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        u32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = T::pack(p[r][2 * e], p[r][2 * e + 1]);
        w[r] = __builtin_bit_cast(bf16x8, x);
        sum[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w[r], sum[r], 0, 0, 0);
      }
#pragma unroll
      for (int n = 0; n < CPL; ++n) {
        const bf16x8 x = T::operand(v, n);
#pragma unroll
        for (int r = 0; r < RT; ++r) o[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w[r], o[r][n], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < NS; ++i) sum[r][0] += p[r][i];
      T::template values<RT, S>(o, v, p);
    }
  }

  // After the tiles t0, t0 + 1, .. < t1: a row's outputs are infinite or NaN where it sees such a
  // value in a masked tile.  channel(c, i): of output o[.][c][i]
  template <typename F>
  __device__ __forceinline__ void settle(const ChunkArgs& a, const ChunkWork& w, const AT* vb, F&& channel) {
    if (bad0 > bad1) return;
    const int P = 1 << a.p.shift;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int c = 0; c < CPL; ++c) {
        floatx4 s = floatx4{};
#pragma unroll 1
        for (int j = bad0 * KEYS; j < min((bad1 + 1) * KEYS, w.s.len); ++j) {
          const int page = paged_page(a.p, w.b, j >> a.p.shift);
          if (page < 0 || !(chunk_window(1u, pos[r], a.window, j) & 1u)) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int ch = channel(c, i);
            const float y = ch < a.dh ? T::value(vb + page * a.p.sp + (j & (P - 1)) * a.p.ss + ch) : 0.f;
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
    if constexpr (BF16) return sum[r][0];
    float2 x = lanes_x16(sum[r][0]);
    x = lanes_x32(x.x + x.y);
    return x.x + x.y;
  }
};

// Row rr of the block's sequence and kv head: its place in the output, in units of dh.
__device__ __forceinline__ int64_t chunk_row(const ChunkArgs& a, const ChunkWork& w, int rr) {
  const int G = a.H / a.Hkv;
  return (int64_t)(w.s.start + rr / G) * a.H + w.hk * G + rr % G;
}

// Few rows: bound by the reads of keys and values, which go straight from memory to the registers
// of the wave that uses them, the next tile's keys on their way during the softmax.  Each of the
// 4 waves takes a run of the block's tiles; their sums meet in LDS.
template <typename AT, int DH, int RT, bool FULL>
__global__ void __launch_bounds__(256, DH* RT <= 128 ? 3 : 1) paged_few_kernel(ChunkArgs a) {
  using Rows = ChunkRows<AT, DH, RT>;
  using T = typename Rows::T;
  constexpr int KEYS = T::KEYS, CPL = T::CPL;
  constexpr int ROWS = 16 * RT, LD = DH + 4;
  __shared__ float xm[4][ROWS], xl[4][ROWS];
  __shared__ float xo[4][ROWS][LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, g = lane >> 4;
  ChunkWork w;
  if (!chunk_work<KEYS, ROWS>(a, w)) return;
  const AT* kb = reinterpret_cast<const AT*>(a.k) + w.hk * a.p.sh;
  const AT* vb = reinterpret_cast<const AT*>(a.v) + w.hk * a.p.sh;
  const float sc = fabsf(a.scale) * 1.4426950408889634f;
  Rows rows;
  typename T::K k;
  typename T::V v;
  PageIds ids;
  ids.start(a, w);
  TileAt<KEYS> now, next;
  // the lane's places within a group of eight keys
  const int64_t k_at = (m & 7) * a.p.ss, v_at = 4 * (g & 1) * a.p.ss;
  auto load_k = [&](const TileAt<KEYS>& at) {
#pragma unroll
    for (int t = 0; t < T::KT; ++t) T::template load_k_row<FULL>(k, t, kb + (m < 8 ? at.off[2 * t] : at.off[2 * t + 1]) + k_at, g, a.dh);
  };
  const int each = (w.t1 - w.t0 + 3) / 4, end = min(w.t1, w.t0 + (wave + 1) * each);
  int t = w.t0 + wave * each;
  if (t < end) {
    now.find(a, ids, t * KEYS);
    load_k(now);
  }
  rows.template start<FULL>(a, w, w.r0, lane);
  for (; t < end; ++t) {
#pragma unroll
    for (int h = 0; h < T::KT; ++h) {
      const AT* row = vb + (g < 2 ? now.off[2 * h] : now.off[2 * h + 1]) + v_at;
#pragma unroll
      for (int e = 0; e < 4; ++e) T::template load_v_row<FULL>(v, 4 * h + e, row + e * a.p.ss, m, a.dh);
    }
    rows.scores(k);
    if (t + 1 < end) {
      next.find(a, ids, (t + 1) * KEYS);
      load_k(next);
    }
    const bool mask = rows.masked(now.present, a.window, t * KEYS);
    rows.soften(now.present, a.window, t * KEYS, mask, g, sc);
    rows.add(v, mask, t);
    now = next;
  }
  rows.settle(a, w, vb, [&](int c, int i) { return T::channel(c, 4 * g + i); });

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
  constexpr int PER = 256 / ROWS;  // threads of a row
  const int c0 = 4 * (tid % PER), row = tid / PER;
  if (row >= w.R - w.r0) return;
  float mx = -INFINITY, l = 0.f, f[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) mx = fmaxf(mx, xm[u][row]);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    f[u] = xm[u][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((xm[u][row] - mx) * sc);
    // (a row whose scores are all NaN has no maximum, but its sum is NaN and stays)
    l += xm[u][row] == -INFINITY ? xl[u][row] : xl[u][row] * f[u];
  }
  const int64_t out_row = chunk_row(a, w, w.r0 + row), part_row = out_row * a.splits + w.split;
  if (tid % PER == 0 && w.ns > 1) a.part_ml[part_row] = make_float2(mx, l);
  for (int c = c0; c < a.dh; c += 4 * PER) {
    floatx4 x = floatx4{};
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] += rescaled(xo[u][row][c + i], f[u]);
    if (w.ns > 1) *reinterpret_cast<floatx4*>(a.part_o + part_row * a.dh + c) = x;
    else attn_store<AT>(a.out, out_row * a.dh + c, x, l);
  }
}

// Many rows (bf16): NW waves of 32 (dh <= 128) or 16 rows each share the keys and values, which
// come through LDS by DMA, two tiles ahead.  A tile is 32 rows of DH channels for keys and as many
// for values; 16-byte piece c of key j lies at piece c ^ (j % 16 or less), so that both the reads
// of one piece of 16 keys and those of all pieces of a key spread over the banks.
template <int DH, int NW, bool FULL>
__global__ void __launch_bounds__(64 * NW, 2) paged_chunk_kernel(ChunkArgs a) {
  constexpr int RT = DH == 256 ? 1 : 2;
  using Rows = ChunkRows<uint16_t, DH, RT>;
  using T = typename Rows::T;
  constexpr int CPL = T::CPL, ROWS = 16 * RT * NW;
  constexpr int PIECES = DH / 8, SWZ = PIECES < 16 ? PIECES - 1 : 15;  // 16-byte pieces of a row
  constexpr int KPD = 64 / PIECES;                                       // keys of a DMA
  constexpr int TILE = 32 * DH, STAGES = 3;                             // elements of a key or value tile
  __shared__ __align__(16) uint16_t buf[STAGES][2][TILE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, g = lane >> 4;
  ChunkWork w;
  if (!chunk_work<32, ROWS>(a, w)) return;
  const uint16_t* kb = reinterpret_cast<const uint16_t*>(a.k) + w.hk * a.p.sh;
  const uint16_t* vb = reinterpret_cast<const uint16_t*>(a.v) + w.hk * a.p.sh;
  const float sc = fabsf(a.scale) * 1.4426950408889634f;
  const uint32_t lds0 = lds_offset(&buf[0][0][0]);
  const int last_piece = a.dh / 8 - 1;
  Rows rows;
  rows.template start<FULL>(a, w, w.r0 + 16 * RT * wave, lane);
  PageIds ids;
  ids.start(a, w);
  // A DMA of a wave fills 1 KB, KPD keys.  Every wave fetches the same keys and values, KD times
  // (width 64 in 8 waves: once, keys or values).  A wave's keys lie within a group of eight.
  constexpr int KD = DH / 16 / NW, DMAS = KD ? 2 * KD : 1;
  auto fetch = [&](int t) {
    const uint32_t to = lds0 + (uint32_t)((t - w.t0) % STAGES * 4 * TILE);
    TileAt<32> at;
    at.find(a, ids, 32 * t);
    auto from = [&](int part) {
      const int j = part * KPD + lane / PIECES, c = (lane % PIECES) ^ (j & SWZ), u = part * KPD / 8;
      const int64_t off = u == 0 ? at.off[0] : (u == 1 ? at.off[1] : (u == 2 ? at.off[2] : at.off[3]));
      return off + (j & 7) * a.p.ss + 8 * (FULL ? c : min(c, last_piece));
    };
    if constexpr (KD > 0) {
#pragma unroll
      for (int i = 0; i < KD; ++i) {
        const int part = i * NW + wave;
        const int64_t off = from(part);
        dma16(kb + off, to + part * 1024);
        dma16(vb + off, to + 2 * TILE + part * 1024);
      }
    } else {
      const int part = wave % (NW / 2);
      dma16((wave < NW / 2 ? kb : vb) + from(part), to + (wave < NW / 2 ? 0 : 2 * TILE) + part * 1024);
    }
    return at.present;
  };
  dma_wait_all();  // the queries are here: from now on only the DMAs count as loads in flight
  uint32_t present[3] = {};  // of this tile and the next two
  if (w.t0 < w.t1) present[0] = fetch(w.t0);
  if (w.t0 + 1 < w.t1) present[1] = fetch(w.t0 + 1);
  for (int t = w.t0; t < w.t1; ++t) {
    // tile t has landed, and every wave is done with tile t - 1, whose place tile t + 2 takes
    if (t + 1 < w.t1) dma_wait_barrier<DMAS>();
    else dma_wait_barrier<0>();
    if (t + 2 < w.t1) present[2] = fetch(t + 2);
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
    const bool mask = rows.masked(present[0], a.window, 32 * t);
    rows.soften(present[0], a.window, 32 * t, mask, g, sc);
    rows.add(v, mask, t);
    present[0] = present[1];
    present[1] = present[2];
  }
  rows.settle(a, w, vb, [&](int c, int i) { return 16 * c + 4 * g + i; });

#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = rows.row_sum(r);
    const int rr = w.r0 + 16 * (RT * wave + r) + m;
    if (rr >= w.R) continue;
    const int64_t out_row = chunk_row(a, w, rr), part_row = out_row * a.splits + w.split;
    if (g == 0 && w.ns > 1) a.part_ml[part_row] = make_float2(rows.top[r], l);
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
      const int ch = 16 * c + 4 * g;  // of four consecutive outputs
      if (!FULL && ch >= a.dh) continue;
      if (w.ns > 1) *reinterpret_cast<floatx4*>(a.part_o + part_row * a.dh + ch) = rows.o[r][c];
      else attn_store<uint16_t>(a.out, out_row * a.dh + ch, rows.o[r][c], l);
    }
  }
}

// A wave per row (new token, head): its splits onto their common maximum, in order.  Groups of
// dh / 4 lanes, four channels each, take every ng-th split; their sums meet by shuffles.
template <typename AT>
__global__ void __launch_bounds__(256) paged_join_kernel(ChunkArgs a, int keys, int block_rows) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= (int64_t)a.p.N * a.H) return;
  const int n = (int)(r / a.H), h = (int)(r % a.H), G = a.H / a.Hkv;
  ChunkWork w;
  w.b = last_at_most(a.p.B, n, [&](int b) { return paged_start(a.p, b); });
  if (w.b < 0) return;
  w.s = paged_seq(a.p, w.b);
  if (n - w.s.start >= w.s.rows) return;
  w.R = w.s.rows * G;
  w.split = 0;
  w.r0 = ((n - w.s.start) * G + h % G) / block_rows * block_rows;
  chunk_tiles(a, w, keys, block_rows);
  if (w.ns == 1) return;
  const float sc = fabsf(a.scale) * 1.4426950408889634f;
  const int64_t part = r * a.splits;
  float mx = -INFINITY;
  for (int s = lane; s < w.ns; s += 64) mx = fmaxf(mx, a.part_ml[part + s].x);
  mx = wave_max(mx);
  const int per = a.dh / 4, ng = 64 / per, grp = lane / per, c = 4 * (lane % per);
  float l = 0.f;
  floatx4 x = floatx4{};
  for (int s = grp; grp < ng && s < w.ns; s += ng) {
    const float2 ml = a.part_ml[part + s];
    const floatx4 o = *reinterpret_cast<const floatx4*>(a.part_o + (part + s) * a.dh + c);
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml.x - mx) * sc);
    // (a row whose scores are all NaN has no maximum, but its sum is NaN and stays)
    l += ml.x == -INFINITY ? ml.y : ml.y * f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += rescaled(o[i], f);
  }
  floatx4 y = x;
  float total = l;
  for (int i = 1; i < ng; ++i) {
    total += __shfl(l, (lane + i * per) & 63);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += __shfl(x[e], (lane + i * per) & 63);
  }
  if (grp == 0) attn_store<AT>(a.out, r * a.dh + c, y, total);
}

// Tiles, row blocks and splits of a call, and its workspace.
struct ChunkPlan {
  int dhp;  // kernel width: 64, 128 or 256
  int rt;   // row tiles of a wave of paged_few_kernel, or 0:
  int nw;   // waves of paged_chunk_kernel
  int rows, row_blocks, splits, min_tiles;
  size_t o_off, bytes;
};

ChunkPlan chunk_plan(int N, int B, int H, int Hkv, int dh, spider_dtype dtype) {
  ChunkPlan p{};
  const bool bf16 = dtype == SPIDER_BF16;
  const int64_t G = H / Hkv, R = N * G;  // rows of a kv head, R / B of an average sequence
  p.dhp = dh <= 64 ? 64 : (dh <= 128 ? 128 : 256);
  const int wave_rows = p.dhp == 256 ? 16 : 32;
  int64_t target;
  if (!bf16 || R <= (int64_t)B * wave_rows) {
    p.rt = R <= (int64_t)B * 16 || p.dhp == 256 ? 1 : 2;
    p.rows = 16 * p.rt;
    target = 768;
  } else {
    // (width 256 has no registers for two waves per SIMD)
    p.nw = R <= (int64_t)B * 2 * wave_rows ? 2 : (R <= (int64_t)B * 4 * wave_rows || p.dhp == 256 ? 4 : 8);
    p.rows = wave_rows * p.nw;
    target = p.dhp == 256 ? 256 : 256 * 8 / p.nw;
  }
  p.row_blocks = (int)(R / p.rows) + B;
  p.min_tiles = 8;
  const int64_t blocks = Hkv * std::max<int64_t>(B, R / p.rows);
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(target / blocks, 128));
  size_t off = 0;
  if (p.splits > 1) {
    const size_t rows = (size_t)N * H * p.splits;
    p.o_off = align_up(rows * sizeof(float2), 256);
    off = align_up(p.o_off + rows * dh * sizeof(float), 256);
  }
  p.bytes = off;
  return p;
}

unsigned chunk_blocks(const ChunkArgs& a) { return (unsigned)(a.Hkv * a.splits) * (unsigned)a.row_blocks; }

template <typename AT, int DH, int RT>
void launch_few(const ChunkArgs& a, hipStream_t st) {
  if (a.dh == DH) paged_few_kernel<AT, DH, RT, true><<<chunk_blocks(a), 256, 0, st>>>(a);
  else paged_few_kernel<AT, DH, RT, false><<<chunk_blocks(a), 256, 0, st>>>(a);
}

template <int DH, int NW>
void launch_chunk(const ChunkArgs& a, hipStream_t st) {
  if (a.dh == DH) paged_chunk_kernel<DH, NW, true><<<chunk_blocks(a), 64 * NW, 0, st>>>(a);
  else paged_chunk_kernel<DH, NW, false><<<chunk_blocks(a), 64 * NW, 0, st>>>(a);
}

template <typename AT, int DH>
spider_status run_chunk(const ChunkArgs& a, const ChunkPlan& p, hipStream_t st) {
  ProfScope ps(KC_PAGED_ATTN, st);
  if (p.rt == 1) launch_few<AT, DH, 1>(a, st);
  if constexpr (DH <= 128)
    if (p.rt == 2) launch_few<AT, DH, 2>(a, st);
  if constexpr (sizeof(AT) == 2) {
    if (p.nw == 2) launch_chunk<DH, 2>(a, st);
    if (p.nw == 4) launch_chunk<DH, 4>(a, st);
    if constexpr (DH <= 128)
      if (p.nw == 8) launch_chunk<DH, 8>(a, st);
  }
  SPIDER_LAUNCHED("paged_attention");
  if (a.splits > 1) {
    paged_join_kernel<AT><<<(unsigned)(((int64_t)a.p.N * a.H + 3) / 4), 256, 0, st>>>(a, AttnTile<AT, DH>::KEYS, p.rows);
    SPIDER_LAUNCHED("paged_join");
  }
  return SPIDER_OK;
}

template <typename AT>
spider_status run_chunk(const ChunkArgs& a, const ChunkPlan& p, hipStream_t st) {
  return p.dhp == 64 ? run_chunk<AT, 64>(a, p, st) : (p.dhp == 128 ? run_chunk<AT, 128>(a, p, st) : run_chunk<AT, 256>(a, p, st));
}

bool chunk_shape_ok(int N, int B, int H, int Hkv, int dh, spider_dtype dtype) {
  return N >= 1 && B >= 1 && B <= kPagedMaxB && H >= 1 && H <= 65535 && Hkv >= 1 && H % Hkv == 0 && dh >= 1 && dh <= kPagedMaxDh &&
         (int64_t)N * H < (1 << 24) && (int64_t)Hkv * B < (1 << 22) && (dtype == SPIDER_BF16 || dtype == SPIDER_F32);
}

}  // namespace
}  // namespace spider

using namespace spider;

extern "C" size_t spider_paged_attention_workspace_size(int N, int B, int H, int Hkv, int dh, spider_dtype dtype) {
  return chunk_shape_ok(N, B, H, Hkv, dh, dtype) ? chunk_plan(N, B, H, Hkv, dh, dtype).bytes : 0;
}

extern "C" spider_status spider_paged_attention(int N, int H, int Hkv, int dh, const void* q, int64_t q_stride,
                                                const spider_paged_cache* cache, spider_dtype dtype, float scale, int window,
                                                void* out, void* workspace, size_t workspace_bytes, spider_stream stream) {
  clear_error();
  SPIDER_REQUIRE(q && out, SPIDER_ERR_INVALID_ARG, "spider_paged_attention: null pointer");
  SPIDER_REQUIRE(dtype == SPIDER_BF16 || dtype == SPIDER_F32, SPIDER_ERR_INVALID_ARG, "spider_paged_attention: bad dtype");
  SPIDER_REQUIRE(N >= 1 && H >= 1 && Hkv >= 1 && dh >= 1, SPIDER_ERR_INVALID_ARG, "spider_paged_attention: sizes must be positive");
  SPIDER_REQUIRE(window >= 0 && std::isfinite(scale), SPIDER_ERR_INVALID_ARG, "spider_paged_attention: window must not be negative, scale finite");
  SPIDER_REQUIRE(H % Hkv == 0, SPIDER_ERR_SHAPE, "spider_paged_attention: %d heads over %d kv heads", H, Hkv);
  ChunkArgs a{};
  const spider_status s = paged_check("spider_paged_attention", cache, N, Hkv, dh, dtype, false, &a.p);
  if (s != SPIDER_OK) return s;
  // blocks of the largest launch (a grid holds 2^24 blocks of 256 threads)
  SPIDER_REQUIRE(chunk_shape_ok(N, cache->B, H, Hkv, dh, dtype), SPIDER_ERR_UNSUPPORTED, "spider_paged_attention: N * H reaches 2^24, B * Hkv 2^22, or H 65536");
  const int64_t per16 = dtype == SPIDER_BF16 ? 8 : 4;
  if (N == 1) q_stride = 0;
  SPIDER_REQUIRE(q_stride % per16 == 0 && q_stride >= 0, SPIDER_ERR_INVALID_ARG, "spider_paged_attention: q_stride must be a multiple of 16 bytes");
  SPIDER_REQUIRE((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) % 16 == 0, SPIDER_ERR_INVALID_ARG,
                 "spider_paged_attention: q and out must be 16-byte aligned");
  const ChunkPlan p = chunk_plan(N, cache->B, H, Hkv, dh, dtype);
  SPIDER_REQUIRE(p.bytes == 0 || (workspace && workspace_bytes >= p.bytes), SPIDER_ERR_WORKSPACE,
                 "spider_paged_attention: workspace of %zu bytes needed, %zu given", p.bytes, workspace ? workspace_bytes : 0);
  SPIDER_REQUIRE(p.bytes == 0 || reinterpret_cast<uintptr_t>(workspace) % 256 == 0, SPIDER_ERR_INVALID_ARG,
                 "spider_paged_attention: workspace must be 256-byte aligned");
  a.q = q, a.k = cache->k, a.v = cache->v, a.out = out, a.qs = q_stride;
  a.H = H, a.Hkv = Hkv, a.dh = dh, a.window = window, a.scale = scale;
  a.row_blocks = p.row_blocks, a.splits = p.splits, a.min_tiles = p.min_tiles;
  if (p.splits > 1) {
    a.part_ml = reinterpret_cast<float2*>(workspace);
    a.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + p.o_off);
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  return dtype == SPIDER_BF16 ? run_chunk<uint16_t>(a, p, st) : run_chunk<float>(a, p, st);
}
