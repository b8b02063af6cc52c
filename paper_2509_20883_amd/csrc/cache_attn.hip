// Attention over the paged 8-bit cache (gfx950): few new queries against long
// histories, the whole of them or listed pages.
//
//   s_ij = cap(scale q_i.k_j) - slope_h |p_i - j|, p_i = i + len - Lq
//   out_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij), k_j = s_k code, v_j = s_v code
//
// One pass over the keys with the running maximum and sum of the softmax. A wave
// takes 32 rows (tokens times the query heads of a key head), one per lane
// column, against 32 keys at a time, and loads both sides of those keys from the
// page straight into the registers that feed the matrix instructions: codes are
// exact in bf16, so only the page's two scales are left to multiply, one into
// the scores and one into the probabilities. fp32 queries and probabilities are
// three bf16 pieces each, which carry their 24 bits through the same
// instructions. The next keys are on their way while a step is computed; no LDS
// and no barrier until the waves' results are joined.
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

template <int N>
__device__ inline void split(const float (&x)[8], bf16x8 (&f)[N]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = pack_bf16(r[2 * e], r[2 * e + 1]);
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
__device__ inline void load8(const uint16_t* p, bool in, bf16x8 (&f)[1]) {
  f[0] = bf16x8{};
  if (in) f[0] = *reinterpret_cast<const bf16x8*>(p);
}
__device__ inline void load8(const float* p, bool in, bf16x8 (&f)[3]) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = 0.0f;
  if (in) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = a[e];
      x[4 + e] = b[e];
    }
  }
  split(x, f);
}
__device__ inline void pieces_of(const uint16_t (&x)[8], bf16x8 (&f)[1]) {
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  u16x8 w;
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = x[e];
  f[0] = __builtin_bit_cast(bf16x8, w);
}
__device__ inline void pieces_of(const float (&x)[8], bf16x8 (&f)[3]) { split(x, f); }

constexpr int kPartBlocks = 8;

// Where a row tile stands and which blocks of 32 keys its sequence has for it.
struct TileAt {
  int s, token0, row0;  // row0: the tile's first row (of the sequence, or of the token's heads where pages are listed)
  int rows, lk, lq;     // rows: of the sequence (of the token)
  int64_t start;
  int closed, end;      // tokens in full pages, tokens that any row of the tile sees
  int blocks, per, parts;  // blocks of 32 keys in full pages; per: of a part
};

// False: no such tile.
__device__ inline bool tile_at(const CacheAttn& a, int64_t unit, int tile_rows, TileAt& t) {
  const CacheArgs& c = a.c;
  int64_t tile;
  if (a.list) {
    const int parts = (a.group + tile_rows - 1) / tile_rows;
    const int64_t u = unit / parts;
    t.row0 = static_cast<int>(unit - u * parts) * tile_rows;
    if (c.pad > 0) {
      if (u >= c.rows) return false;
      t.s = static_cast<int>(u / c.pad);
      tile = u - t.s * c.pad;
    } else {
      t.s = find_seq(c.off, c.seqs, 1, 1, u, tile);
    }
  } else if (c.pad > 0) {
    const int64_t per = (c.pad * a.group + tile_rows - 1) / tile_rows;
    t.s = static_cast<int>(unit / per);
    tile = unit - t.s * per;
    if (t.s >= c.seqs) return false;
  } else {
    t.s = find_seq(c.off, c.seqs, a.group, tile_rows, unit, tile);
  }
  if (tile < 0) return false;
  const SeqSpan q = seq_span(c.off, t.s, c.pad, c.rows);
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
    const int64_t r0 = tile * tile_rows, all = c.pad > 0 ? c.pad * a.group : static_cast<int64_t>(q.len) * a.group;
    if (r0 >= all) return false;
    t.row0 = static_cast<int>(r0);
    t.token0 = 0;
    t.rows = q.len * a.group;
    last = t.row0 < t.rows ? div_group(min(t.row0 + tile_rows, t.rows) - 1, a.group) : -1;
  }
  t.end = last < 0 || t.rows == 0 ? 0 : a.causal ? max(0, min(t.lk, last + t.lk - t.lq + 1)) : t.lk;
  if (t.end == 0) t.blocks = 0;
  else if (a.list) t.blocks = a.count << (c.plog - 5);
  else t.blocks = (min(t.end, t.closed) + kCacheBlock - 1) / kCacheBlock;
  // at least eight blocks to a part: fewer are not worth its way through memory
  const int share = (t.blocks + a.splits - 1) / a.splits;
  t.per = max(kPartBlocks, (share + kPartBlocks - 1) / kPartBlocks * kPartBlocks);
  t.parts = max(1, (t.blocks + t.per - 1) / t.per);
  return true;
}

// A lane's output columns and its row's running maximum, the height above it at
// which it moves, and sum of the softmax, in base 2.
template <int M, int HD>
struct AttnState {
  typename Shape<M>::acc acc[HD / M];
  float m, move, l;
};

struct RowParams {
  int limit, pos, least;  // keys the row sees; least: of the wave's rows
  float slope, scale, cap;
};

// The lane's 16 keys from position j on into the softmax: p comes as the products
// of the codes and leaves as probabilities times vs. masked: some lane's row may
// not see some key of the step.
template <typename T, int M, int HD>
__device__ __forceinline__ void soften(AttnState<M, HD>& st, float (&p)[16], const RowParams& r, bool capped, bool sloped,
                                       float ks, float vs, int j, bool masked) {
  float c = r.scale * kLog2e * ks;
  if (capped) {
    c = r.cap * kLog2e;
    tanh_scores<T>(p, r.scale / r.cap * ks);
  }
  if (!sloped) {
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = p[i] * c - st.m;
  } else {
    const float dist = static_cast<float>(j - r.pos);
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = p[i] * c - (r.slope * fabsf(dist + static_cast<float>(i)) + st.m);
  }
  if (masked) {
    const int left = r.limit - j;
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = i < left ? p[i] : -INFINITY;
  }
  float top = p[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, p[i]);
  top = Shape<M>::column_max(top);
  // the running maximum moves only when a score passes it by 2^8
  if (__any(top > st.move)) {
    const bool up = top > st.move;
    const float by = up ? top : 0.0f;
    const float alpha = st.move == -INFINITY ? 0.0f : exp2_hw(-by);
    st.m += by;
    st.move = up ? 8.0f : st.move;
    st.l *= alpha;
#pragma unroll
    for (int i = 0; i < HD / M; ++i) st.acc[i] *= alpha;
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] -= by;
  }
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = exp2_hw(p[i]);
    sum += p[i];
    p[i] *= vs;
  }
  st.l += sum;
}

// Waves of a SIMD that the registers are kept down for.
template <typename T, int HD, int M>
constexpr int kResident = HD <= 32 ? 3 : HD <= 64 && (M == 16 || sizeof(T) == 2) ? 3 : HD * sizeof(T) <= 256 || M == 16 ? 2 : 1;

// Tiles of WR M rows: WR waves along the rows, WK along the keys, each taking steps
// of 1024 / M keys.
template <typename T, bool E4M3, int HD, int M, int WR, int WK>
__global__ __launch_bounds__(WR* WK* kWave, (kResident<T, HD, M>)) void k_cache_attn(const CacheAttn a) {
  typedef Shape<M> S;
  constexpr int G = kWave / M;                       // lane groups
  constexpr int B = 16 * G / kCacheBlock;            // blocks of a step
  constexpr int KT = 16 * G / M;                     // key tiles of a step
  constexpr int KC = HD < 16 * G ? 1 : HD / (16 * G);  // 16-column chunks of a key per lane
  constexpr int DT = HD / M, NP = Pieces<T>::N, kRows = M * WR;
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wr = wave % WR, wk = wave / WR, grp = lane / M, col = lane % M;
  const int64_t b = a.block0 + blockIdx.x;
  const int part = static_cast<int>(b % a.splits);
  const int kvh = static_cast<int>(b / a.splits % c.hkv);
  const int64_t unit = b / a.splits / c.hkv;
  TileAt t;
  if (!tile_at(a, unit, kRows, t) || part >= t.parts) return;  // block-uniform
  const int b0 = part * t.per, b1 = min(b0 + t.per, t.blocks);
  const bool joined = t.parts > 1;

  const int r = t.row0 + wr * M + col;
  const bool live = r < t.rows;
  RowOf me;
  if (a.list) {
    me.token = t.token0;
    me.head = kvh * a.group + r;
  } else {
    me = row_of(r, kvh, a.group);
  }
  RowParams rp;
  rp.limit = !live ? 0 : a.causal ? max(0, min(t.lk, me.token + t.lk - t.lq + 1)) : t.lk;
  rp.pos = me.token + t.lk - t.lq;
  // keys that every row of the wave sees: limits do not fall along the rows
  const int least = __builtin_amdgcn_readfirstlane(rp.limit);
  rp.slope = a.slopes && live ? a.slopes[me.head] * kLog2e : 0.0f;
  rp.scale = a.scale;
  rp.cap = a.cap;
  const bool capped = a.cap > 0.0f, sloped = a.slopes != nullptr;

  bf16x8 qf[2 * KC][NP];
  {
    const T* q = static_cast<const T*>(a.q.p) + (t.start + me.token) * a.q.row + me.head * a.q.head;
#pragma unroll
    for (int i = 0; i < 2 * KC; ++i) {
      const int d0 = i / 2 * 16 * G + grp * 16 + (i & 1) * 8;
      load8(q + d0, live && d0 < c.d, qf[i]);
    }
  }
  AttnState<M, HD> st;
#pragma unroll
  for (int i = 0; i < DT; ++i) st.acc[i] = typename S::acc{};
  st.m = 0.0f;
  st.move = -INFINITY;
  st.l = 0.0f;

  // the lane's row of a key tile, so that scores 0 .. 15 of group g are keys 16 g ..
  auto key_of = [&](int tile) { return M == 32 ? ((col >> 2) & 1) * 16 + (col >> 3) * 4 + (col & 3) : (col >> 2) * 16 + tile * 4 + (col & 3); };
  const int64_t page_bytes = static_cast<int64_t>(HD) << c.plog;
  const int sub_mask = (1 << (c.plog - 5)) - 1;

  // the wave's steps: n blocks from b0 + wk B on, every WK B
  int pages = -1, firsts = 0;  // of the next blocks, one per lane: page and first token
  auto look = [&](int n) {
    const int64_t mine = n + static_cast<int64_t>(lane / B) * (WK * B) + lane % B;
    int num = -1;
    firsts = 0;
    if (mine < b1) {
      const int at = static_cast<int>(mine) >> (c.plog - 5);
      num = a.list ? a.list[((t.start + t.token0) * c.hkv + kvh) * a.count + at] : at;
      if (num >= t.closed >> c.plog) num = -1;
      firsts = (num << c.plog) + ((static_cast<int>(mine) & sub_mask) << 5);
    }
    pages = cache_page(c, t.s, num);
  };
  // block i of the step at place j (0 .. 64 / B - 1) of those looked up
  auto page_at = [&](int j, int i) { return B == 1 ? __builtin_amdgcn_readlane(pages, j) : __shfl(pages, j * B + i, kWave); };
  auto first_at = [&](int j, int i) { return B == 1 ? __builtin_amdgcn_readlane(firsts, j) : __shfl(firsts, j * B + i, kWave); };

  u32x4 kc[KT][KC], vc[DT];
  float2 scale = make_float2(0.0f, 0.0f);
  auto load_keys = [&](int j) {
    const int i = B == 1 ? 0 : col >> 3;  // the lane's keys lie in one block
    const int page = page_at(j, i), sub = (first_at(j, i) >> 5) & sub_mask;
    const uint8_t* p = c.data + (static_cast<int64_t>(page) * c.hkv + kvh) * 2 * page_bytes;
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
      for (int y = 0; y < KC; ++y) {
        const int chunk = y * G + grp;
        kc[x][y] = u32x4{0, 0, 0, 0};
        if (page >= 0 && (HD >= 16 * G || chunk < HD / 16))
          kc[x][y] = *reinterpret_cast<const u32x4*>(p + (((chunk << c.plog) + sub * kCacheBlock + (key_of(x) & 31)) << 4));
      }
  };
  auto load_values = [&](int j) -> int {  // the lane's first key, or -1
    const int i = B == 1 ? 0 : grp >> 1;
    const int page = page_at(j, i), first = first_at(j, i), sub = (first >> 5) & sub_mask;
    const int64_t at = static_cast<int64_t>(page) * c.hkv + kvh;
    const uint8_t* p = c.data + (at * 2 + 1) * page_bytes;
    scale = make_float2(0.0f, 0.0f);
    if (page >= 0) scale = reinterpret_cast<const float2*>(c.scales)[at];
#pragma unroll
    for (int x = 0; x < DT; ++x) {
      vc[x] = u32x4{0, 0, 0, 0};
      if (page >= 0) vc[x] = *reinterpret_cast<const u32x4*>(p + (((sub * 2 + (grp & 1)) * HD + x * M + col) << 4));
    }
    return page >= 0 ? first + (grp & 1) * 16 : -1;
  };

  const int stride = WK * B;
  int n = b0 + wk * B, j = 0;
  if (n < b1) {
    look(n);
    load_keys(0);
  }
  for (; n < b1; n += stride) {
    const int key0 = load_values(j);
    float p[16];
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      typename S::acc sc = {};
#pragma unroll
      for (int y = 0; y < KC; ++y)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 kf[1] = {codes8<E4M3>(kc[x][y][2 * u], kc[x][y][2 * u + 1])};
          sc = mma_pieces<M>(kf, qf[2 * y + u], sc);
        }
#pragma unroll
      for (int i = 0; i < 16 / KT; ++i) p[x * (16 / KT) + i] = sc[i];
    }
    // the next keys into the same registers, under the softmax and the second product
    if (n + stride < b1) {
      j = j + 1 == kWave / B ? 0 : j + 1;
      if (j == 0) look(n + stride);
      load_keys(j);
    }
    RowParams now = rp;
    now.limit = key0 < 0 ? INT32_MIN / 2 : rp.limit;  // a page that is not there
    const bool masked = !__all(key0 >= 0 && key0 + 16 <= least);
    soften<T>(st, p, now, capped, sloped, scale.x, scale.y, key0, masked);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = p[8 * u + e];
      bf16x8 pf[NP];
      split(y, pf);
#pragma unroll
      for (int x = 0; x < DT; ++x) {
        const bf16x8 vf[1] = {codes8<E4M3>(vc[x][2 * u], vc[x][2 * u + 1])};
        st.acc[x] = mma_pieces<M>(vf, pf, st.acc[x]);
      }
    }
  }
  // the open page, with the last part
  const int slot = cache_slot(c, t.s), held = t.lk - t.closed, most = t.end - t.closed;
  if (part == t.parts - 1 && slot >= 0) {
    const T* kp = static_cast<const T*>(c.open) + open_at(c, slot, t.closed >> c.plog, kvh, 0);
    const T* vp = kp + (static_cast<int64_t>(c.d) << c.plog);
    for (int k0 = wk * 16 * G; k0 < most; k0 += WK * 16 * G) {
      float p[16];
#pragma unroll
      for (int x = 0; x < KT; ++x) {
        const int k = k0 + key_of(x);
        typename S::acc sc = {};
#pragma unroll
        for (int y = 0; y < 2 * KC; ++y) {
          const int d0 = y / 2 * 16 * G + grp * 16 + (y & 1) * 8;
          bf16x8 kf[NP];
          load8(kp + k * c.d + d0, k < held && d0 < c.d, kf);
          sc = mma_pieces<M>(kf, qf[y], sc);
        }
#pragma unroll
        for (int i = 0; i < 16 / KT; ++i) p[x * (16 / KT) + i] = sc[i];
      }
      soften<T>(st, p, rp, capped, sloped, 1.0f, 1.0f, t.closed + k0 + grp * 16, true);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = p[8 * u + e];
        bf16x8 pf[NP];
        split(y, pf);
#pragma unroll
        for (int x = 0; x < DT; ++x) {
          T z[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = k0 + grp * 16 + u * 8 + e;
            z[e] = T(0);
            if (k < held && x * M + col < c.d) z[e] = vp[k * c.d + x * M + col];
          }
          bf16x8 vf[NP];
          pieces_of(z, vf);
          st.acc[x] = mma_pieces<M>(vf, pf, st.acc[x]);
        }
      }
    }
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
    const int64_t at = ((unit * c.hkv + kvh) * a.splits + part) * kRows + wr * M + col;
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
  T* out = static_cast<T*>(a.out) + ((t.start + me.token) * a.hq + me.head) * c.d;
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

// Joins the splits of a row: a block per query token and head, threads four
// columns and a share of the splits each.
//   m = max m_c,  l = sum l_c 2^(m_c - m),  out = sum acc_c 2^(m_c - m) / l
template <typename T, int NT>
__global__ __launch_bounds__(NT) void k_cache_join(const CacheAttn a, int tile_rows, int64_t block0) {
  __shared__ float4 sh_o[NT];
  __shared__ float sh_l[NT], sh_m[NT / kWave];
  const CacheArgs& c = a.c;
  const int64_t b = block0 + blockIdx.x;
  const int head = static_cast<int>(b % a.hq), kvh = head / a.group;
  const int64_t u = b / a.hq;
  int s;
  int64_t token;
  if (c.pad > 0) {
    s = static_cast<int>(u / c.pad);
    token = u - s * c.pad;
  } else {
    s = find_seq(c.off, c.seqs, 1, 1, u, token);
  }
  const SeqSpan q = seq_span(c.off, s, c.pad, c.rows);
  if (token < 0 || token >= q.len) return;  // rows past a padded sequence's end are written
  int64_t unit;
  int at;
  if (a.list) {
    const int tiles = (a.group + tile_rows - 1) / tile_rows, r = head - kvh * a.group;
    unit = u * tiles + r / tile_rows;
    at = r % tile_rows;
  } else {
    const int64_t r = token * a.group + head - kvh * a.group;
    const int64_t first = c.pad > 0 ? s * ((c.pad * a.group + tile_rows - 1) / tile_rows)
                                    : tile_base(c.off, s, a.group, tile_rows);
    unit = first + r / tile_rows;
    at = static_cast<int>(r % tile_rows);
  }
  TileAt t;
  if (!tile_at(a, unit, tile_rows, t) || t.parts == 1) return;  // written
  const int parts = t.parts;
  const int64_t slot0 = (unit * c.hkv + kvh) * a.splits * tile_rows + at;

  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  float m = -INFINITY;
  for (int i = threadIdx.x; i < parts; i += NT) {
    const float2 x = ml[slot0 + static_cast<int64_t>(i) * tile_rows];
    m = fmaxf(m, x.y == 0.0f ? -INFINITY : x.x);
  }
#pragma unroll
  for (int i = kWave / 2; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor(m, i, kWave));
  if ((threadIdx.x & (kWave - 1)) == 0) sh_m[threadIdx.x / kWave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) m = fmaxf(m, sh_m[w]);
  const float base = m == -INFINITY ? 0.0f : m;

  const int quads = c.d / 4;  // at most 32
  const int shares = NT / quads, quad = threadIdx.x % quads, share = threadIdx.x / quads;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float l = 0.0f;
  if (share < shares) {
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
  if (share > 0) return;
  for (int k = 1; k < shares; ++k) {
    const float4 y = sh_o[k * quads + quad];
    l += sh_l[k * quads + quad];
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

constexpr int64_t kMostBlocks = int64_t(1) << 21;

template <typename T, bool E4M3, int HD>
hipError_t run(CacheAttn a, hipStream_t s) {
  const int64_t blocks = a.units * a.c.hkv * a.splits;
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {
    a.block0 = b;
    const unsigned now = static_cast<unsigned>(std::min(blocks - b, kMostBlocks));
    if (a.tile_rows == 16) k_cache_attn<T, E4M3, HD, 16, 1, 4><<<now, 4 * kWave, 0, s>>>(a);
    else if (a.tile_rows == 32) k_cache_attn<T, E4M3, HD, 32, 1, 4><<<now, 4 * kWave, 0, s>>>(a);
    else k_cache_attn<T, E4M3, HD, 32, 4, 1><<<now, 4 * kWave, 0, s>>>(a);
  }
  if (a.splits > 1) {
    const int64_t rows = (a.c.pad > 0 ? a.c.rows : a.c.rows + a.c.seqs) * a.hq;
    for (int64_t b = 0; b < rows; b += kMostBlocks) {
      const unsigned now = static_cast<unsigned>(std::min(rows - b, kMostBlocks));
      if (a.splits > 32) k_cache_join<T, 1024><<<now, 1024, 0, s>>>(a, a.tile_rows, b);
      else k_cache_join<T, 128><<<now, 128, 0, s>>>(a, a.tile_rows, b);
    }
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

constexpr int64_t kSplitBlocks = 1024;
constexpr int64_t kLeastChunk = 256;
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
  const int tile_rows = a->tile_rows = most_rows <= 16 ? 16 : most_rows <= 32 || a->list ? 32 : 128;
  if (a->list) {
    a->units = (c.pad > 0 ? c.rows : c.rows + c.seqs) * ((a->group + tile_rows - 1) / tile_rows);
  } else if (c.pad > 0) {
    a->units = c.seqs * ((c.pad * a->group + tile_rows - 1) / tile_rows);
  } else {
    a->units = c.rows * a->group / tile_rows + c.seqs;
  }
  int64_t keys = c.width << c.plog;
  if (max_len > 0) keys = std::min(keys, max_len);
  if (a->list) keys = (static_cast<int64_t>(a->count) << c.plog) + (1 << c.plog);
  const int64_t blocks = a->units * c.hkv;
  int64_t splits = std::min((kSplitBlocks + blocks - 1) / blocks, keys / kLeastChunk);
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
