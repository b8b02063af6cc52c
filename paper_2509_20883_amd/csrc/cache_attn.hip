// Attention over the paged 8-bit cache (gfx950): few new queries against long
// histories, the whole of them or listed pages.
//
//   s_ij = cap(scale q_i.k_j) - slope_h |p_i - j|, p_i = i + len - Lq
//   out_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij), k_j = s_k code, v_j = s_v code
//
// One pass over the keys with the running maximum and sum of the softmax. A wave
// takes 32 or 16 rows (tokens times the query heads of a key head), one per lane
// column, against 32 keys at a time. Codes are exact in bf16, so only the page's two
// scales are left to multiply, one into the scores and one into the probabilities
// (the latter, a power of two in e4m3, by the conversion itself). fp32 queries and
// probabilities are three bf16 pieces each, which carry their 24 bits through the
// same instructions; with bf16 queries the probabilities are rounded to bf16, the
// type of the products (two pieces of each, as exact as the output's own rounding:
// 4096 rows over 16384 keys 296 -> 400 us, a token of 256 users 74 -> 77). Scores,
// maxima, sums and outputs are fp32.
//
// Few rows (16 or 32 a tile): the four waves of a block lie along the keys, and each
// loads both sides of its keys from the page straight into the registers that feed
// the matrix instructions, the next 32 on their way while these are computed; LDS
// only joins the waves' results. Bound by reading the pages: without any products
// the loads alone take as long (64 x 32768 keys of 128 206 us, 208 with them), and
// whole rows of 256 bytes gathered at random reach 5.4 TB/s. One token of 256 users
// with 1 to 4096 keys of 128 in 2 heads (257 MB) 67 us, 4 rows over 1,000,003 keys of 64
// (256 MB) 52: 15 to 25 us of that are there at any size (the chain from a row's
// sequence to its length, its pages and their first bytes, code that is not in the
// caches yet, and the end of the longest sequence, which has as many parts as the
// shortest).
//
// Many rows: tiles of 128, a wave 32 of them, over the same keys; the operands are
// made once a block into LDS. Bound by the vector instructions around the products
// (conversions, exponentials, the running maximum: vector unit 45% busy, matrix unit
// 38%, the rest waits between the two): 4096 rows over 16384 keys of 128, 8 query heads,
// 294 us and 22 to join, 810 TFLOP/s over the visible keys in a pass; in i8 333 a pass,
// in fp32 817.
//
// The open page's tokens, at most page_len - 1 of a sequence, are read in the
// model's type.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_common.h"

#pragma clang fp contract(fast)

namespace rs {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Pieces of a value of the model's type as bf16 numbers: bf16 is one, fp32
// (24 bits) three.
template <typename T>
struct Pieces {
  static constexpr int N = sizeof(T) == 2 ? 1 : 3;
};

// ANY: the values may pass bf16's largest, which a first piece then stays at (rounded, it
// would be infinite and the others NaN).
template <bool ANY, int N>
__device__ inline void split(const float (&x)[8], bf16x8 (&f)[N]) {
  constexpr float kMost = 0x1.FEp127f;
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool cut = ANY && n == 0 && N > 1;
      w[e] = cut ? pack_bf16(__builtin_amdgcn_fmed3f(r[2 * e], -kMost, kMost), __builtin_amdgcn_fmed3f(r[2 * e + 1], -kMost, kMost))
                 : pack_bf16(r[2 * e], r[2 * e + 1]);
      if (n + 1 < N) {
        r[2 * e] -= __uint_as_float(w[e] << 16);
        r[2 * e + 1] -= __uint_as_float(w[e] & 0xFFFF0000u);
      }
    }
    f[n] = __builtin_bit_cast(bf16x8, w);
  }
}

// The matrix instruction of M x M results: M = 32 for many rows, 16 where a tile
// has at most 16, which leaves half the registers. A lane's group (lane / M) holds
// slots 8 group .. 8 group + 7 of the product and, of a result, 4 consecutive rows
// of column lane % M at a time.
template <int M>
struct Shape;
template <>
struct Shape<32> {
  typedef f32x16 acc;
  __device__ static inline acc mma(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  __device__ static inline float column_max(float x) { return other_half_max(x); }
  __device__ static inline float column_sum(float x) { return other_half_sum(x); }
};
template <>
struct Shape<16> {
  typedef f32x4 acc;
  __device__ static inline acc mma(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  __device__ static inline float column_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return other_half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
  }
  __device__ static inline float column_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return other_half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  }
};

// The sum of the products of two sets of pieces, the smallest (below 2^-24 of
// the whole) left out.
template <int M, int NA, int NB>
__device__ inline typename Shape<M>::acc mma_pieces(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], typename Shape<M>::acc c) {
  constexpr int kMost = NA > NB ? NA : NB;
#pragma unroll
  for (int i = NA - 1; i >= 0; --i)
#pragma unroll
    for (int j = NB - 1; j >= 0; --j)
      if (i + j < kMost) c = Shape<M>::mma(a[i], b[j], c);
  return c;
}

// Eight values of a row as pieces, from global memory.
__device__ inline void load8(const uint16_t* p, bf16x8 (&f)[1]) { f[0] = *reinterpret_cast<const bf16x8*>(p); }
__device__ inline void load8(const float* p, bf16x8 (&f)[3]) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  split<true>(x, f);
}
__device__ inline void pieces_of(const uint16_t (&x)[8], bf16x8 (&f)[1]) {
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  u16x8 w;
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = x[e];
  f[0] = __builtin_bit_cast(bf16x8, w);
}
__device__ inline void pieces_of(const float (&x)[8], bf16x8 (&f)[3]) { split<true>(x, f); }

constexpr int kKeyWaves = 4;  // of a block whose waves lie along the keys
constexpr int kPartBlocks = 2 * kKeyWaves;

// Where a row tile stands and which blocks of 32 keys its sequence has for it.
struct TileAt {
  int s, token0, row0;  // row0: the tile's first row (of the sequence, or of the token's heads where pages are listed)
  int rows, lk, lq;     // rows: of the sequence (of the token)
  int64_t start;
  int closed, end;         // tokens in full pages, tokens that any row of the tile sees
  int blocks, per, parts;  // blocks of 32 keys in full pages; per: of a part
};

// A tile of sequence t.s: number `tile` of its tiles of 1 << log rows, or where
// pages are listed rows t.row0 on of its token `tile`. False: no such tile.
__device__ inline bool tile_of(const CacheAttn& a, const SeqSpan& q, int64_t tile, int log, TileAt& t) {
  const CacheArgs& c = a.c;
  t.start = q.start;
  t.lq = q.len;
  t.lk = cache_len(c, t.s);
  t.closed = t.lk >> c.plog << c.plog;
  int last;  // token of the tile's last row
  if (a.list) {
    if (tile >= (c.pad > 0 ? c.pad : int64_t(q.len))) return false;
    t.token0 = last = static_cast<int>(tile);
    t.rows = tile < q.len ? a.group : 0;
  } else {
    const int64_t r0 = tile << log, all = (c.pad > 0 ? c.pad : int64_t(q.len)) * a.group;
    if (r0 >= all) return false;
    t.row0 = static_cast<int>(r0);
    t.token0 = 0;
    t.rows = q.len * a.group;
    last = t.row0 < t.rows ? div_group(min(t.row0 + (1 << log), t.rows) - 1, a.group) : -1;
  }
  t.end = last < 0 || t.rows == 0 ? 0 : a.causal ? max(0, min(t.lk, last + t.lk - t.lq + 1)) : t.lk;
  if (t.end == 0) t.blocks = 0;
  else if (a.list) t.blocks = a.count << (c.plog - 5);
  else t.blocks = (min(t.end, t.closed) + kCacheBlock - 1) / kCacheBlock;
  // a part is at least two steps of every wave: fewer are not worth its way through memory
  const int share = static_cast<int>(static_cast<uint32_t>(t.blocks + a.splits - 1) / static_cast<uint32_t>(a.splits));
  t.per = max(kPartBlocks, (share + kPartBlocks - 1) / kPartBlocks * kPartBlocks);
  t.parts = max(1, static_cast<int>(static_cast<uint32_t>(t.blocks + t.per - 1) / static_cast<uint32_t>(t.per)));
  return true;
}

// Tile number `unit` of all. Fewer than 2^31 of them.
__device__ inline bool tile_at(const CacheAttn& a, uint32_t unit, int log, TileAt& t) {
  const CacheArgs& c = a.c;
  int64_t tile;
  const int tile_rows = 1 << log;
  if (a.list) {
    const uint32_t tiles = static_cast<uint32_t>(a.group + tile_rows - 1) >> log;
    const uint32_t u = tiles == 1 ? unit : unit / tiles;
    t.row0 = static_cast<int>(unit - u * tiles) << log;
    if (c.pad > 0) {
      t.s = static_cast<int>(u / static_cast<uint32_t>(c.pad));
      tile = u - static_cast<uint32_t>(t.s) * static_cast<uint32_t>(c.pad);
    } else {
      t.s = find_tile(c.off, c.seqs, 1, 0, u, tile);
    }
  } else if (c.pad > 0) {
    const uint32_t tiles = static_cast<uint32_t>(c.pad * a.group + tile_rows - 1) >> log;
    t.s = static_cast<int>(unit / tiles);
    tile = unit - static_cast<uint32_t>(t.s) * tiles;
  } else {
    t.s = find_tile(c.off, c.seqs, a.group, log, unit, tile);
  }
  if (tile < 0 || t.s >= c.seqs) return false;
  return tile_of(a, seq_span(c.off, t.s, c.pad, c.rows), tile, log, t);
}

// A lane's output columns and its row's running maximum, the height above it at
// which it moves, and sum of the softmax, in base 2.
template <int M, int HD>
struct AttnState {
  typename Shape<M>::acc acc[HD / M];
  float m, move, l;
};

template <typename T>
__device__ inline void capped_scores(float (&x)[16], float scale) {
  tanh_scores<T>(x, scale);
}
template <typename T>
__device__ inline void capped_scores(float (&x)[8], float scale) {
  float y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = x[i & 7];  // the second eight fall away as the same
  tanh_scores<T>(y, scale);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = y[i];
}

struct RowParams {
  int limit, pos, least;  // keys the row sees; least: of the wave's rows
  float slope, scale, cap;
};

// The lane's NS keys from position j on into the softmax: p comes as the products
// of the codes and leaves as probabilities, SCALED times vs. masked: some lane's row
// may not see some key of the step.
template <typename T, bool SCALED, int M, int HD, int NS>
__device__ __forceinline__ void soften(AttnState<M, HD>& st, float (&p)[NS], const RowParams& r, bool capped, bool sloped,
                                       float ks, float vs, int j, bool masked) {
  float c = r.scale * kLog2e * ks;
  if (capped) {
    c = r.cap * kLog2e;
    capped_scores<T>(p, r.scale / r.cap * ks);
  }
  // Distances are taken from the lane's nearest key, `near` away, and that one's term with
  // the maximum: two large numbers near each other where the key counts at all, so that
  // their sum is exact (from the row's position at once, a key next to the row after one
  // a million back was off by their distance's last bit: fp32 rows by 4e-4 of their norm).
  float near = 0.0f;
  if (sloped) {
    const int dist = j - r.pos;
    const float e = static_cast<float>(min(max(dist, 1 - NS), 0));
    near = r.slope * static_cast<float>(max(max(dist, 1 - NS - dist), 0));
#pragma unroll
    for (int i = 0; i < NS; ++i) p[i] = p[i] * c - r.slope * fabsf(e + static_cast<float>(i));
    c = 1.0f;
  }
  if (masked) {
    const int left = r.limit - j;
#pragma unroll
    for (int i = 0; i < NS; ++i) p[i] = i < left ? p[i] : -INFINITY;
    c = c == 0.0f ? 0x1p-149f : c;  // a product that is gone in fp32 keeps them out all the same
  }
  float top = p[0];
#pragma unroll
  for (int i = 1; i < NS; ++i) top = fmaxf(top, p[i]);
  top = Shape<M>::column_max(top * c - (near + st.m));
  // the running maximum moves only when a score passes it by 2^8
  if (__any(top > st.move)) {
    const bool up = top > st.move;
    const float m = up ? st.m + top : st.m;
    const float alpha = st.move == -INFINITY ? 0.0f : exp2_hw(st.m - m);
    st.m = m;
    st.move = up ? 8.0f : st.move;
    st.l *= alpha;
#pragma unroll
    for (int i = 0; i < HD / M; ++i) st.acc[i] *= alpha;
  }
  const float past = near + st.m;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    p[i] = exp2_hw(p[i] * c - past);
    sum += p[i];
    if (SCALED) p[i] *= vs;
  }
  st.l += sum;
}

// Waves of a SIMD that the registers are kept down for.
template <typename T, int HD, int M>
constexpr int kResident = M == 16 ? (sizeof(T) == 4 ? (HD <= 64 ? 3 : 2) : HD <= 64 ? 4 : 3) : HD <= 64 ? (sizeof(T) == 2 ? 4 : 3) : sizeof(T) == 2 ? 3 : 1;

__device__ inline float lane_value(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// Tiles of WR M rows: WR waves along the rows, WK along the keys, each taking 32
// keys at a time.
template <typename T, bool E4M3, int HD, int M, int WR, int WK>
__global__ __launch_bounds__(WR* WK* kWave, (kResident<T, HD, M>)) void k_cache_attn(const CacheAttn a) {
  typedef Shape<M> S;
  constexpr int G = kWave / M;                         // lane groups
  constexpr int NS = kCacheBlock / G;                  // keys of a group: consecutive ones
  constexpr int KT = kCacheBlock / M;                  // key tiles of a step
  constexpr int KC = HD < 16 * G ? 1 : HD / (16 * G);  // 16-column chunks of a key per lane
  constexpr int DT = HD / M, NU = NS / 8, NP = Pieces<T>::N, kRows = M * WR;
  typedef uint32_t codes_t __attribute__((ext_vector_type(NS / 4)));
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wr = wave % WR, wk = wave / WR, grp = lane / M, col = lane % M;
  // the last tiles, which see the most keys under a causal mask, first
  const uint32_t unit = a.unit0 + gridDim.x - 1 - blockIdx.x;
  const int kvh = blockIdx.y, part = blockIdx.z;
  TileAt t;
  if (!tile_at(a, unit, kRows == 16 ? 4 : kRows == 32 ? 5 : 7, t) || part >= t.parts) return;  // block-uniform
  const int b0 = part * t.per, b1 = min(b0 + t.per, t.blocks);
  const bool joined = t.parts > 1;

  const int r = t.row0 + wr * M + col;
  const bool live = r < t.rows;
  // rows that are not there stand for the last: what they get is not written
  const int r_in = live ? r : max(t.rows - 1, 0);
  RowOf me;
  if (a.list) {
    me.token = t.token0;
    me.head = kvh * a.group + r_in;
  } else {
    me = row_of(r_in, kvh, a.group);
  }
  RowParams rp;
  rp.limit = a.causal ? max(0, min(t.lk, me.token + t.lk - t.lq + 1)) : t.lk;
  rp.pos = me.token + t.lk - t.lq;
  // keys that every row of the wave sees: limits do not fall along the rows
  const int least = __builtin_amdgcn_readfirstlane(rp.limit);
  rp.slope = a.slopes ? a.slopes[me.head] * kLog2e : 0.0f;
  rp.scale = a.scale;
  rp.cap = a.cap;
  const bool capped = a.cap > 0.0f, sloped = a.slopes != nullptr;

  // The rows as an operand. Those of 128 bf16 columns lie in LDS, in the order of the
  // lanes: their 32 registers are what keeps a third wave off a SIMD.
  constexpr bool kRowsInLds = M == 32 && WR == 1 && HD == 128 && sizeof(T) == 2;
  __shared__ __align__(16) char q_rows[kRowsInLds ? WR * 2 * KC * kWave * 16 : 16];
  bf16x8* const my_rows = reinterpret_cast<bf16x8*>(q_rows) + wr * 2 * KC * kWave + lane;
  bf16x8 qf[kRowsInLds ? 1 : 2 * KC][NP];
  {
    const T* q = static_cast<const T*>(a.q.p) + (t.start + me.token) * a.q.row + me.head * a.q.head;
#pragma unroll
    for (int i = 0; i < 2 * KC; ++i) {
      const int d0 = i / 2 * 16 * G + grp * 16 + (i & 1) * 8;
      const bool in = d0 < c.d && t.rows > 0;
      bf16x8 f[NP];
#pragma unroll
      for (int n = 0; n < NP; ++n) f[n] = bf16x8{};
      if (t.rows > 0) load8(q + (in ? d0 : 0), f);
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        if (!in) f[n] = bf16x8{};
        if (!kRowsInLds) qf[i][n] = f[n];
      }
      if (kRowsInLds && wk == 0) my_rows[i * kWave] = f[0];
    }
    if (kRowsInLds) __syncthreads();
  }
  auto with_rows = [&](const auto& kf, int i, typename S::acc sc) {
    if constexpr (kRowsInLds) {
      const bf16x8 f[1] = {my_rows[i * kWave]};
      return mma_pieces<M>(kf, f, sc);
    } else {
      return mma_pieces<M>(kf, qf[i], sc);
    }
  };
  AttnState<M, HD> st;
#pragma unroll
  for (int i = 0; i < DT; ++i) st.acc[i] = typename S::acc{};
  st.m = 0.0f;
  st.move = -INFINITY;
  st.l = 0.0f;

  // the lane's row of a key tile, so that a lane's results are keys NS grp + 0 ..
  auto key_of = [&](int tile) {
    return M == 32 ? ((col >> 2) & 1) * 16 + (col >> 3) * 4 + (col & 3) : (col >> 2) * 8 + tile * 4 + (col & 3);
  };
  const int64_t page_bytes = static_cast<int64_t>(HD) << c.plog;
  const int sub_mask = (1 << (c.plog - 5)) - 1;

  // of the wave's next 64 blocks, one per lane: page, first token and scales (a
  // load of a step's scales in the step would make it wait for the next keys too)
  int pages = -1, firsts = 0;
  float2 scales = make_float2(0.0f, 0.0f);
  const int part_blocks = b1 - b0;
  auto look = [&](int s) {
    const int64_t step = s + static_cast<int64_t>(lane) * WK;
    int num = -1;
    firsts = 0;
    if (step < part_blocks) {
      const int mine = b0 + static_cast<int>(step), at = mine >> (c.plog - 5);
      num = a.list ? a.list[((t.start + t.token0) * c.hkv + kvh) * a.count + at] : at;
      if (num >= t.closed >> c.plog) num = -1;
      firsts = (num << c.plog) + ((mine & sub_mask) << 5);
    }
    pages = cache_page(c, t.s, num);
    if (pages >= 0) scales = reinterpret_cast<const float2*>(c.scales)[static_cast<int64_t>(pages) * c.hkv + kvh];
    if (scales.y != scales.y) scales.x = scales.y;  // the conversion of e4m3 takes a scale's exponent alone
  };

  u32x4 kc[KT][KC];
  codes_t vc[DT];
  float2 scale = make_float2(0.0f, 0.0f);
  // a page that is not there stands as page 0, and its step is left out; so is that of
  // a page whose tokens are lost (keys' scale 0, looked at where the scales are needed)
  auto load_keys = [&](int j) {
    const int page = max(__builtin_amdgcn_readlane(pages, j), 0), sub = (__builtin_amdgcn_readlane(firsts, j) >> 5) & sub_mask;
    const uint8_t* p = c.data + (static_cast<int64_t>(page) * c.hkv + kvh) * 2 * page_bytes;
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
      for (int y = 0; y < KC; ++y) {
        const uint32_t chunk = HD >= 16 * G ? y * G + grp : min(grp, HD / 16 - 1);  // past the head: q is 0 there
        const uint32_t at = ((chunk << c.plog) + sub * kCacheBlock + key_of(x)) << 4;
        kc[x][y] = *reinterpret_cast<const u32x4*>(p + at);
      }
  };
  auto load_values = [&](int j) -> int {  // the step's first key, or -1
    const int page = __builtin_amdgcn_readlane(pages, j), first = __builtin_amdgcn_readlane(firsts, j);
    const int64_t at = static_cast<int64_t>(max(page, 0)) * c.hkv + kvh;
    const uint8_t* p = c.data + (at * 2 + 1) * page_bytes;
    const uint32_t chunk = ((first >> 5) & sub_mask) * 2 + NS * grp / 16;
    scale = make_float2(lane_value(scales.x, j), lane_value(scales.y, j));
#pragma unroll
    for (int x = 0; x < DT; ++x) {
      const uint32_t to = ((chunk * HD + x * M + col) << 4) + NS * grp % 16;
      vc[x] = *reinterpret_cast<const codes_t*>(p + to);
    }
    return page >= 0 && scale.x != 0.0f ? first : -1;
  };
  auto scores_coded = [&](float (&p)[NS]) {
    if (kRowsInLds) asm volatile("" ::: "memory");  // the rows are read again, not kept
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      typename S::acc sc = {};
#pragma unroll
      for (int y = 0; y < KC; ++y)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 kf[1] = {codes8<E4M3>(kc[x][y][2 * u], kc[x][y][2 * u + 1], 1.0f)};
          sc = with_rows(kf, 2 * y + u, sc);
        }
#pragma unroll
      for (int i = 0; i < NS / KT; ++i) p[x * (NS / KT) + i] = sc[i];
    }
  };
  auto output_coded = [&](const bf16x8 (&pf)[NU][NP]) {
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int x = 0; x < DT; ++x) {
        const bf16x8 vf[1] = {codes8<E4M3>(vc[x][2 * u], vc[x][2 * u + 1], scale.y)};
        st.acc[x] = mma_pieces<M>(vf, pf[u], st.acc[x]);
        if (x % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // no operands are made ahead
      }
  };

  // the wave's steps: every WK-th, those of full pages first, then with the last
  // part those of the open page
  const int slot = cache_slot(c, t.s), held = t.lk - t.closed;
  const int most = part == t.parts - 1 && slot >= 0 ? t.end - t.closed : 0;
  const int full_steps = c.pages > 0 ? part_blocks : 0;
  const int steps = full_steps + (most > 0 ? (most + kCacheBlock - 1) / kCacheBlock : 0);
  const T* open = static_cast<const T*>(c.open) + (most > 0 ? open_at(c, slot, t.closed >> c.plog, kvh, 0) : 0);
  // tokens past the page's last stand for it and columns past the head for the
  // first: their scores are masked, their products with q are with 0
  auto scores_open = [&](float (&p)[NS], int k0) {
    int last = held - 1;
    asm volatile("" : "+s"(last));  // or the addresses are made ahead of the loop and kept
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const uint32_t row = min(k0 + key_of(x), last) * c.d;
      typename S::acc sc = {};
#pragma unroll
      for (int y = 0; y < 2 * KC; ++y) {
        const int d0 = y / 2 * 16 * G + grp * 16 + (y & 1) * 8;
        bf16x8 kf[NP];
        load8(open + (row + (d0 < c.d ? d0 : 0)), kf);
        sc = with_rows(kf, y, sc);
      }
#pragma unroll
      for (int i = 0; i < NS / KT; ++i) p[x * (NS / KT) + i] = sc[i];
    }
  };
  auto output_open = [&](const bf16x8 (&pf)[NU][NP], int k0) {
    int last = held - 1;
    asm volatile("" : "+s"(last));
    const char* v = reinterpret_cast<const char*>(open + (static_cast<int64_t>(c.d) << c.plog));
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int x = 0; x < DT; ++x) {
        T z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t at = min(k0 + grp * NS + u * 8 + e, last) * c.d + min(x * M + col, c.d - 1);
          z[e] = *reinterpret_cast<const T*>(v + at * static_cast<uint32_t>(sizeof(T)));
        }
        bf16x8 vf[NP];
        pieces_of(z, vf);
        st.acc[x] = mma_pieces<M>(vf, pf[u], st.acc[x]);
        if (x % (M / 8) == M / 8 - 1) __builtin_amdgcn_sched_barrier(0);  // not all loads at once: they spill
      }
  };
  auto pieces = [&](const float (&p)[NS], bf16x8 (&pf)[NU][NP]) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = p[8 * u + e];
      split<false>(y, pf[u]);
    }
  };

  // Few rows: a block lives for a few steps, and what it fetches of the kernel's
  // code counts as much as its data (the open page in a loop of its own: token of
  // 256 users 77 us, so 67), so both kinds of steps share one softmax.
  constexpr bool kShared = M == 16;
  int s = wk;
  if constexpr (WR > 1) {
    // Waves along the rows read the same keys: each makes the operands of its share
    // of them, once, into LDS, a step ahead. (Every wave by itself: 4096 rows over
    // 16384 keys 338 us in e4m3 and 435 in i8: bound by those conversions.)
    constexpr int kItems = KC + DT, kEach = (kItems + WR - 1) / WR;  // 16-byte loads of a step, of a wave
    constexpr int kFrags = 2 * KC + NU * DT;
    __shared__ __align__(16) bf16x8 operands[2][kFrags * kWave];
    struct Step {
      int first;  // below 0: a page that is not there
      float ks, vs;
    };
    u32x4 raw[kEach];
    auto fetch = [&](int n) {
      const int j = n & (kWave - 1);
      if (j == 0) look(n);
      const int page = __builtin_amdgcn_readlane(pages, j), first = __builtin_amdgcn_readlane(firsts, j);
      const int sub = (first >> 5) & sub_mask;
      const uint8_t* p = c.data + (static_cast<int64_t>(max(page, 0)) * c.hkv + kvh) * 2 * page_bytes;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int item = wr * kEach + k;
        if (item < KC) {
          const uint32_t chunk = HD >= 16 * G ? item * G + grp : min(grp, HD / 16 - 1);
          raw[k] = *reinterpret_cast<const u32x4*>(p + (((chunk << c.plog) + sub * kCacheBlock + key_of(0)) << 4));
        } else if (item < kItems) {
          raw[k] = *reinterpret_cast<const u32x4*>(p + page_bytes + (((sub * 2 + grp) * HD + (item - KC) * M + col) << 4));
        }
      }
      const float ks = lane_value(scales.x, j);
      return Step{page >= 0 && ks != 0.0f ? first : -1, ks, lane_value(scales.y, j)};
    };
    auto place = [&](int n, const Step& x) {
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int item = wr * kEach + k;
        if (item >= kItems) continue;
        const bool keys = item < KC;
        bf16x8* to = operands[n & 1] + (keys ? 2 * item : 2 * KC + item - KC) * kWave + lane;
        const float vs = keys ? 1.0f : x.vs;
        to[0] = codes8<E4M3>(raw[k][0], raw[k][1], vs);
        to[(keys ? 1 : DT) * kWave] = codes8<E4M3>(raw[k][2], raw[k][3], vs);
      }
    };
    const int furthest = __builtin_amdgcn_readlane(rp.limit, M - 1);  // keys that any row of the wave sees
    Step now{}, next{};
    if (full_steps > 0) {
      now = fetch(0);
      place(0, now);
      if (full_steps > 1) next = fetch(1);
    }
    for (s = 0; s < full_steps; ++s) {
      __syncthreads();  // this step's operands are there, the other place has been read
      const Step at = now;
      now = next;
      if (s + 1 < full_steps) place(s + 1, next);
      if (s + 2 < full_steps) next = fetch(s + 2);
      if (at.first < 0 || at.first >= furthest) continue;
      const bf16x8* from = operands[s & 1] + lane;
      typename S::acc sc = {};
#pragma unroll
      for (int i = 0; i < 2 * KC; ++i) {
        const bf16x8 kf[1] = {from[i * kWave]};
        sc = mma_pieces<M>(kf, qf[i], sc);
      }
      float p[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) p[i] = sc[i];
      soften<T, !E4M3>(st, p, rp, capped, sloped, at.ks, at.vs, at.first + grp * NS, at.first + kCacheBlock > least);
      bf16x8 pf[NU][NP];
      pieces(p, pf);
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int x = 0; x < DT; ++x) {
          const bf16x8 vf[1] = {from[(2 * KC + u * DT + x) * kWave]};
          st.acc[x] = mma_pieces<M>(vf, pf[u], st.acc[x]);
        }
    }
  } else {
    int j = 0;
    if (wk < full_steps) {
      look(wk);
      load_keys(0);
    }
    for (; s < (kShared ? steps : full_steps); s += WK) {
      const bool coded = !kShared || s < full_steps;  // wave-uniform
      const int k0 = (s - full_steps) * kCacheBlock;
      int key0 = t.closed + k0;
      float p[NS];
      if (coded) {
        key0 = load_values(j);
        scores_coded(p);
        // the next keys into the same registers, under the softmax and the second product
        if (s + WK < full_steps) {
          j = j + 1 == kWave ? 0 : j + 1;
          if (j == 0) look(s + WK);
          load_keys(j);
        }
        if (key0 < 0) continue;  // a page that is not there
      } else {
        scale = make_float2(1.0f, 1.0f);
        scores_open(p, k0);
      }
      const bool masked = !coded || key0 + kCacheBlock > least;
      soften<T, !E4M3>(st, p, rp, capped, sloped, scale.x, scale.y, key0 + grp * NS, masked);
      bf16x8 pf[NU][NP];
      pieces(p, pf);
      if (coded) output_coded(pf);
      else output_open(pf, k0);
    }
  }
  if (!kShared)
    for (; s < steps; s += WK) {
      const int k0 = (s - full_steps) * kCacheBlock;
      float p[NS];
      scores_open(p, k0);
      soften<T, false>(st, p, rp, capped, sloped, 1.0f, 1.0f, t.closed + k0 + grp * NS, true);
      bf16x8 pf[NU][NP];
      pieces(p, pf);
      output_open(pf, k0);
    }

  st.l = S::column_sum(st.l);
  float m = st.m, l = st.l;
  constexpr int R = M == 32 ? 16 : 4;  // a lane's registers of a tile
  if constexpr (WK > 1) {
    // the waves' parts: m = max m_w, acc = sum acc_w 2^(m_w - m), l alike
    constexpr int kPart = DT * R * kWave * sizeof(float);
    __shared__ __align__(16) char parts[WK / 2 * WR * kPart];
    __shared__ float2 sh_ml[WK][WR][M];
    if (grp == 0) sh_ml[wk][wr][col] = make_float2(m, l);
    __syncthreads();
    float base = -INFINITY;
#pragma unroll
    for (int w = 0; w < WK; ++w) base = fmaxf(base, sh_ml[w][wr][col].y == 0.0f ? -INFINITY : sh_ml[w][wr][col].x);
    base = base == -INFINITY ? 0.0f : base;
    const float mul = l == 0.0f ? 0.0f : exp2_hw(m - base);
#pragma unroll
    for (int i = 0; i < DT; ++i) st.acc[i] *= mul;
#pragma unroll
    for (int w = WK / 2; w >= 1; w /= 2) {  // the upper half of the waves hand theirs to the lower half
      f32x4* at = reinterpret_cast<f32x4*>(parts + (wk % w * WR + wr) * kPart) + lane;
      if (wk >= w && wk < 2 * w)
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int e = 0; e < R / 4; ++e)
            at[(i * (R / 4) + e) * kWave] =
                f32x4{st.acc[i][4 * e], st.acc[i][4 * e + 1], st.acc[i][4 * e + 2], st.acc[i][4 * e + 3]};
      __syncthreads();
      if (wk < w)
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int e = 0; e < R / 4; ++e) {
            const f32x4 x = at[(i * (R / 4) + e) * kWave];
#pragma unroll
            for (int y = 0; y < 4; ++y) st.acc[i][4 * e + y] += x[y];
          }
      __syncthreads();
    }
    if (wk > 0) return;
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float2 x = sh_ml[w][wr][col];
      l += x.y == 0.0f ? 0.0f : x.y * exp2_hw(x.x - base);
    }
    m = base;
  }
  // rows of the tile: those of the padded copy past the sequence's end get 0
  const int64_t out_rows = a.list ? a.group : c.pad > 0 ? c.pad * a.group : static_cast<int64_t>(t.rows);
  if (r >= out_rows || (!live && part > 0)) return;
  if (joined && live) {
    const int64_t at = ((static_cast<int64_t>(unit) * c.hkv + kvh) * a.splits + part) * kRows + wr * M + col;
    float* po = a.part_o + at * c.d;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int g = 0; g < R / 4; ++g) {
        const int d0 = i * M + g * 4 * G + grp * 4;
        if (d0 < c.d) store4(po + d0, st.acc[i][4 * g], st.acc[i][4 * g + 1], st.acc[i][4 * g + 2], st.acc[i][4 * g + 3]);
      }
    if (grp == 0) reinterpret_cast<float2*>(a.part_ml)[at] = make_float2(m, l);
    return;
  }
  const bool none = !live || l == 0.0f;  // no key: 0 (a NaN sum stays)
  const float inv = none ? 0.0f : 1.0f / l;
  const RowOf to = a.list ? RowOf{t.token0, kvh * a.group + r} : row_of(r, kvh, a.group);
  T* out = static_cast<T*>(a.out) + ((t.start + to.token) * a.hq + to.head) * c.d;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int g = 0; g < R / 4; ++g) {
      const int d0 = i * M + g * 4 * G + grp * 4;
      if (d0 >= c.d) continue;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = none ? 0.0f : st.acc[i][4 * g + e] * inv;
      store4(out + d0, x[0], x[1], x[2], x[3]);
    }
}

// Joins the parts of a row: NT threads a query token and head, each four columns
// and a share of the parts. Bound by the latency of its loads, one after another:
// the sequence, its length, then maxima, sums and parts together (256 tokens of 8
// heads 6 us). Past 32 parts a block of 1024 threads (4 tokens of 4 heads 10 us).
//   m = max m_c,  l = sum l_c 2^(m_c - m),  out = sum acc_c 2^(m_c - m) / l
template <typename T, int NT>
__global__ __launch_bounds__(NT < kBlock ? kBlock : NT) void k_cache_join(const CacheAttn a) {
  constexpr int kThreads = NT < kBlock ? kBlock : NT, kRows = kThreads / NT;  // rows: heads of one token
  __shared__ float4 sh_o[kThreads];
  __shared__ float sh_l[kThreads], sh_m[kThreads / kWave];
  const CacheArgs& c = a.c;
  const int th = threadIdx.x % NT, row = threadIdx.x / NT;
  const uint32_t u = blockIdx.x;
  TileAt t;
  int64_t token;
  if (c.pad > 0) {
    t.s = static_cast<int>(u / static_cast<uint32_t>(c.pad));
    token = u - static_cast<uint32_t>(t.s) * static_cast<uint32_t>(c.pad);
  } else {
    t.s = find_tile(c.off, c.seqs, 1, 0, u, token);
  }
  const SeqSpan q = seq_span(c.off, t.s, c.pad, c.rows);
  if (token < 0 || token >= q.len) return;  // block-uniform; rows past a padded sequence's end are written
  const int head = min(static_cast<int>(blockIdx.y) * kRows + row, a.hq - 1);
  const bool twice = static_cast<int>(blockIdx.y) * kRows + row >= a.hq;
  const int kvh = static_cast<int>(static_cast<uint32_t>(head) / static_cast<uint32_t>(a.group));
  const int log = a.tile_log, tile_rows = 1 << log;
  uint32_t unit;
  int64_t tile;
  int at;
  if (a.list) {
    const int r = head - kvh * a.group;
    unit = u * (static_cast<uint32_t>(a.group + tile_rows - 1) >> log) + (static_cast<uint32_t>(r) >> log);
    at = r & (tile_rows - 1);
    t.row0 = r - at;
    tile = token;
  } else {
    const int r = static_cast<int>(token) * a.group + head - kvh * a.group;
    const uint32_t first = c.pad > 0 ? static_cast<uint32_t>(t.s) * (static_cast<uint32_t>(c.pad * a.group + tile_rows - 1) >> log)
                                     : static_cast<uint32_t>(max(c.off[t.s], int64_t(0)) * a.group >> log) + t.s;
    tile = static_cast<uint32_t>(r) >> log;
    unit = first + static_cast<uint32_t>(tile);
    at = r & (tile_rows - 1);
  }
  tile_of(a, q, tile, log, t);
  const int parts = t.parts;  // 1: written. A group's heads may lie in two tiles of other ends
  const int64_t slot0 = (static_cast<int64_t>(unit) * c.hkv + kvh) * a.splits * tile_rows + at;

  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  float m = -INFINITY;
  if (parts > 1)
    for (int i = th; i < parts; i += NT) {
      const float2 x = ml[slot0 + static_cast<int64_t>(i) * tile_rows];
      m = fmaxf(m, x.y == 0.0f ? -INFINITY : x.x);
    }
#pragma unroll
  for (int i = kWave / 2; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor(m, i, kWave));
  if constexpr (NT > kWave) {
    if ((threadIdx.x & (kWave - 1)) == 0) sh_m[threadIdx.x / kWave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) m = fmaxf(m, sh_m[w]);
  }
  const float base = m == -INFINITY ? 0.0f : m;

  const uint32_t quads = c.d / 4;  // at most 32
  const int shares = NT / quads, quad = th % quads, share = th / quads;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float l = 0.0f;
  if (share < shares && parts > 1) {
#pragma unroll 4
    for (int i = share; i < parts; i += shares) {
      const int64_t slot = slot0 + static_cast<int64_t>(i) * tile_rows;
      const float2 x = ml[slot];
      const float4 y = *reinterpret_cast<const float4*>(a.part_o + slot * c.d + 4 * quad);
      const float w = x.y == 0.0f ? 0.0f : exp2_hw(x.x - base);
      l += w * x.y;
      o.x += w * y.x;
      o.y += w * y.y;
      o.z += w * y.z;
      o.w += w * y.w;
    }
  }
  sh_o[threadIdx.x] = o;
  sh_l[threadIdx.x] = l;
  __syncthreads();
  if (share > 0 || parts == 1 || twice) return;
  for (int k = 1; k < shares; ++k) {
    const int from = row * NT + k * static_cast<int>(quads) + quad;
    const float4 y = sh_o[from];
    l += sh_l[from];
    o.x += y.x;
    o.y += y.y;
    o.z += y.z;
    o.w += y.w;
  }
  const bool none = l == 0.0f;
  const float inv = none ? 0.0f : 1.0f / l;
  store4(static_cast<T*>(a.out) + ((q.start + token) * a.hq + head) * c.d + 4 * quad, none ? 0.0f : o.x * inv,
         none ? 0.0f : o.y * inv, none ? 0.0f : o.z * inv, none ? 0.0f : o.w * inv);
}

// Fewer than 2^32 threads along an axis of a launch.
constexpr int64_t kMostUnits = int64_t(1) << 21;

template <typename T, bool E4M3, int HD>
hipError_t run(CacheAttn a, hipStream_t s) {
  for (int64_t u = 0; u < a.units; u += kMostUnits) {
    a.unit0 = static_cast<uint32_t>(u);
    const dim3 grid(static_cast<unsigned>(std::min(a.units - u, kMostUnits)), a.c.hkv, a.splits);
    if (a.tile_log == 4) k_cache_attn<T, E4M3, HD, 16, 1, kKeyWaves><<<grid, kKeyWaves * kWave, 0, s>>>(a);
    else if (a.tile_log == 5) k_cache_attn<T, E4M3, HD, 32, 1, kKeyWaves><<<grid, kKeyWaves * kWave, 0, s>>>(a);
    else k_cache_attn<T, E4M3, HD, 32, 4, 1><<<grid, 4 * kWave, 0, s>>>(a);
  }
  if (a.splits > 1) {  // fewer than kSplitBlocks tiles: at most 2^18 rows
    const unsigned n = static_cast<unsigned>(a.c.rows);
    if (a.splits > 32) k_cache_join<T, 1024><<<dim3(n, a.hq), 1024, 0, s>>>(a);
    else k_cache_join<T, kWave><<<dim3(n, (a.hq + 3) / 4), kBlock, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, bool E4M3>
hipError_t run_width(const CacheAttn& a, hipStream_t s) {
  if (a.c.d <= 32) return run<T, E4M3, 32>(a, s);
  if (a.c.d <= 64) return run<T, E4M3, 64>(a, s);
  return run<T, E4M3, 128>(a, s);
}

}  // namespace

// Blocks that a call's keys are split into, measured with pages that come from HBM
// (several caches in turn). One token of 256 users with 1 to 4096 keys: 89 us with 512,
// 82 with 768, 79 with 1536, 80 with 3072: a long sequence's parts have to spread. Few
// row tiles, whose many parts the join has to read: four rows over 1,000,003 keys of 64
// 70 us with 512, 73 with 1024. Listed pages, all rows of like length: a token of 64
// users over 32 pages of 64 41 us with 768, 47 with 1536.
constexpr int64_t kSplitBlocks = 1536, kListBlocks = 768, kFewTileBlocks = 512, kFewTiles = 64;
// Tiles of 128 rows, three blocks a CU: chunks of 33 to 257 queries over 2000 to 8191
// keys 109 us with 256, 80 with 768, 88 with 1024, 89 with 1536; 4096 rows over 16384
// keys 330 with 768, 340 with 1024, 343 with 1536.
constexpr int64_t kWideBlocks = 768;
constexpr int64_t kLeastChunk = 32 * kPartBlocks;
constexpr size_t kMostPartBytes = size_t(256) << 20;

size_t plan_cache_attn(CacheAttn* a, int64_t max_q, int64_t max_len, size_t* ml_at) {
  const CacheArgs& c = a->c;
  a->splits = 1;
  a->units = 0;
  *ml_at = 0;
  if (c.seqs == 0 || c.rows == 0) return 0;
  int64_t most_q = c.pad > 0 ? c.pad : c.rows;
  if (c.pad == 0 && max_q > 0) most_q = std::min(most_q, max_q);
  const int64_t most_rows = a->list ? a->group : most_q * a->group;
  a->tile_log = most_rows <= 16 ? 4 : most_rows <= 32 || a->list ? 5 : 7;
  const int tile_rows = 1 << a->tile_log;
  if (a->list) {
    a->units = c.rows * ((a->group + tile_rows - 1) / tile_rows);
  } else if (c.pad > 0) {
    a->units = c.seqs * ((c.pad * a->group + tile_rows - 1) / tile_rows);
  } else {
    a->units = c.rows * a->group / tile_rows + c.seqs;
  }
  int64_t keys = c.width << c.plog;
  if (max_len > 0) keys = std::min(keys, max_len);
  if (a->list) keys = (static_cast<int64_t>(a->count) << c.plog) + (1 << c.plog);
  const int64_t blocks = a->units * c.hkv;
  const int64_t most = a->tile_log == 7 ? kWideBlocks : blocks < kFewTiles ? kFewTileBlocks : a->list ? kListBlocks : kSplitBlocks;
  int64_t splits = std::min((most + blocks - 1) / blocks, keys / kLeastChunk);
  const size_t one = static_cast<size_t>(blocks) * tile_rows * (c.d + 2) * sizeof(float);
  splits = std::min<int64_t>(splits, kMostPartBytes / one);
  if (splits <= 1) return 0;
  a->splits = static_cast<int>(splits);
  const size_t rows = static_cast<size_t>(blocks) * splits * tile_rows;
  *ml_at = (rows * c.d * sizeof(float) + 255) / 256 * 256;
  return *ml_at + rows * 2 * sizeof(float);
}

hipError_t launch_cache_attn(const CacheAttn& a, bool bf16, bool e4m3, hipStream_t s) {
  if (bf16) return e4m3 ? run_width<uint16_t, true>(a, s) : run_width<uint16_t, false>(a, s);
  return e4m3 ? run_width<float, true>(a, s) : run_width<float, false>(a, s);
}

}  // namespace rs
