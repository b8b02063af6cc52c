// Attention over ragged sequences, backward (gfx950).  With P the forward's
// probabilities, recomputed from the scores and lse:
//
//   dv = P^T dout,  dP = dout v^T,  delta_i = sum_d dout_id out_id
//   ds = P (dP - delta),  dx = ds (1 - tanh^2) scale  (tanh of the capped score)
//   dq = dx k,  dk = dx^T q,  dslope_h = -sum ds |p_i - j|
//
// Two passes, each owning its outputs, so no sum is taken by atomics and
// repeated calls agree bit for bit: one over key tiles for dk and dv, walking
// over the packed rows (all query heads of the key head, so their gradients
// add up in registers), one over row tiles for dq, walking over the keys.  The
// scores and dP are computed in both, seven products instead of five; a single
// pass would need atomics into one of the gradients.
//
// What bounds them: waits, half of the waves' cycles and more in bf16, with two or
// three blocks a CU (the gradients' registers allow no more; one of the small
// shape for rows of 256 bytes, whose tiles take 152 KB).  A step's loads are
// requested a step ahead, but the compiler waits for every load that writes LDS:
// in dk and dv before the step's first read, so that each step pays a trip to
// memory, in dq (bf16) before its first transposed read.  1536 padded sequences
// of 100 to 1024, 2 heads of 64, distances weighed and their slopes' gradient
// taken: dq 727 us, dk and dv 849; 24 documents of 17 to 1500, 16 heads of 128
// over 4, capped: 259 and 469.  The matrix unit is 15 to 20% busy, the vector unit
// 25 to 49%; in fp32 (128 lists of 0 to 400, 4 heads of 32) 32 to 45% and 15%.
#include <hip/hip_runtime.h>

#include "attn_common.h"

#pragma clang fp contract(fast)

namespace rs {
namespace {

// What the pass over keys needs of a row, arrays of q_rows * heads_q words
// written by k_attn_dq: -lse in base 2 (-infinity: no key seen, P = 0), delta,
// the position as an integer (for the mask) and the slope in base 2.
enum : int { kStatLse = 0, kStatDelta = 1, kStatPos = 2, kStatSlope = 3, kStats = 4 };
static_assert(kStats == kAttnStats, "the workspace holds them");

// A word per lane from p + off (bytes; past 2^31: 0) to 64 consecutive words of LDS.
__device__ inline void load_words(const float* p, uint32_t off, float* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
      reinterpret_cast<void*>(static_cast<uint64_t>(hi) << 32 | lo), 0, 0x7FFFFFFF, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)dst, 4, off, 0, 0, 0);
#endif
}

// Four consecutive tile rows' values from LDS.
__device__ inline f32x4 four(const float* p, int r) { return *reinterpret_cast<const f32x4*>(p + r); }

template <typename T, int HD>
constexpr int kResidentBlocks = HD * sizeof(T) > 256 ? 1 : 2;
// The dq pass holds one gradient, and up to 128 bytes a row three blocks fit
// (padded sequences of 560 keys of 64: 990 us with two, 809 with three).
template <typename T, int HD>
constexpr int kResidentRowBlocks = HD * sizeof(T) <= 128 ? 3 : kResidentBlocks<T, HD>;

// How a block of the pass over keys is shaped: KW waves side by side on 32 keys
// each, times RW waves that take turns on the 32-row parts of a step of STEP
// rows and add up their gradients at the end.
//
// Two gradients of 32 keys take HD / 2 + HD / 2 registers a lane.  To leave room
// for two blocks a CU (three up to 128 bytes a row), one in its products while
// another is in its exponentials, the keys stay in LDS as operands, and up to
// 128 bytes a row the values too (padded sequences of 560 keys of 64, dk and dv:
// keys and values in registers, two blocks 1087 us, in LDS, three 978).
//
// Few key tiles (long sequences, many query heads on a key head) are bound by
// the longest one, not by the rate: tiles of 64 keys with more waves along the
// rows then take a quarter (a half) of the time each.
template <typename T, int HD, bool FEW>
struct KeyShape {
  static constexpr int kRow = HD * sizeof(T);
  static constexpr bool kNarrow = kRow <= 128, kWide = kRow > 256;
  static_assert(!FEW || !kWide, "fp32 rows of 128 have one shape");
  static constexpr int KW = FEW ? 2 : 4;
  static constexpr int RW = !FEW ? 1 : kNarrow ? 2 : 4;
  static constexpr int W = KW * RW;       // waves
  // rows per step: 32 for every row wave, and at least a load of 16 bytes for every thread
  static constexpr int STEP = 32 * RW * kRow < W * kWave * 16 ? W * kWave * 16 / kRow : 32 * RW;
  static constexpr int KEYS = 32 * KW;    // keys per block
  static constexpr bool VALUES_IN_LDS = kNarrow;
  static constexpr int BLOCKS = kWide ? 1 : kNarrow ? 3 : 8 / W;  // per CU
};

// dk and dv of a key tile, a wave 32 keys, one per lane column.
template <typename T, int HD, bool FEW>
__global__ __launch_bounds__((KeyShape<T, HD, FEW>::W * kWave), (KeyShape<T, HD, FEW>::BLOCKS * KeyShape<T, HD, FEW>::W / 4)) void k_attn_dkdv(
    const AttnArgs a) {
  typedef KeyShape<T, HD, FEW> C;
  typedef Tile<T, HD> L;
  typedef typename Frag<T>::type F;
  constexpr int KS = HD / 16, DT = HD / 32;
  constexpr int kStep = C::STEP;
  constexpr int kTile = kStep * L::kRowBytes, kKeyTile = C::KEYS * L::kRowBytes;
  // q and dout, two steps of each, then the keys (and values)
  __shared__ __align__(1024) char lds[4 * kTile + (C::VALUES_IN_LDS ? 2 : 1) * kKeyTile];
  char *key_tile = lds + 4 * kTile, *val_tile = key_tile + kKeyTile;
  // of the step's rows, as k_attn_dq left them; 0 where there is no row: its q and dout are 0 too, and add nothing
  constexpr int kStatRows = kStep < kWave ? kWave : kStep;
  // and the row's position from the step's first token on, the same in every step:
  // fp32 then holds the distances of near keys however long the sequence is
  constexpr int kStepPos = kStats;
  __shared__ __align__(16) float stat[2][kStats + 1][kStatRows];

  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int half = lane >> 5, col = lane & 31;
  const int kw = wave % C::KW, rw = wave / C::KW;
  const BlockOf blk = block_of(a, false);
  const int kvh = blk.kvh;
  int s;
  int64_t tile;
  if (a.kv_pad > 0) {
    const uint32_t per = static_cast<uint32_t>((a.kv_pad + C::KEYS - 1) / C::KEYS);
    s = static_cast<uint32_t>(blk.tile) / per;
    tile = blk.tile - static_cast<int64_t>(s) * per;
  } else {
    s = find_seq(a.kv_off, a.seqs, 1, C::KEYS, blk.tile, tile);
  }
  const SeqSpan qs = seq_span(a.q_off, s, a.q_pad, a.q_rows), ks = seq_span(a.kv_off, s, a.kv_pad, a.kv_rows);
  const int64_t out_rows = a.kv_pad > 0 ? a.kv_pad : ks.len;
  if (tile < 0 || tile * C::KEYS >= out_rows) return;  // block-uniform
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;

  const int j0 = static_cast<int>(tile) * C::KEYS;
  const int jw = j0 + kw * 32;  // the wave's first key
  const int j = jw + col;         // the lane's key
  const bool live = j < ks.len;
  F vf[C::VALUES_IN_LDS ? 1 : KS];
  if (!C::VALUES_IN_LDS) {
    const T* v = static_cast<const T*>(a.v.p) + (ks.start + j) * a.v.row + kvh * a.v.head;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int k0 = t * 16 + half * 8;
      vf[t] = zero_frag<T>();
      if (live && k0 < a.d) load_frag(v + k0, vf[t]);
    }
  }
  const float scale2 = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap2 = a.cap * kLog2e;
  const int see_all = a.causal ? prefix : ks.len;  // keys that every row sees

  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) {
    dk[i] = f32x16{};
    dv[i] = f32x16{};
  }
  // the first token that sees the tile's first key
  int first = 0;
  if (a.causal && j0 >= prefix) first = max(0, j0 - (ks.len - qs.len));
  if (j0 >= ks.len) first = qs.len;

  const RowSteps<kStep> steps(a.group);
  RowLoader<T, HD, kStep, C::W> ql, ol;
  ql.init(a.q, qs.start, kvh, a.group, a.d);
  ol.init(HeadRows{a.dout, int64_t(a.hq) * a.d, a.d}, qs.start, kvh, a.group, a.d);
  // Step n: token first + n / parts * tokens, head n % parts * kStep of the group.
  const int n_steps = first < qs.len ? (qs.len - first + steps.tokens - 1) / steps.tokens * steps.parts : 0;
  // the row that the thread loads the statistics of, 64 rows a wave
  const int stat_row = threadIdx.x;
  const int stat_up = steps.parts > 1 ? 0 : div_group(stat_row, a.group);
  const uint32_t stat_off = static_cast<uint32_t>(stat_up * a.hq + stat_row - stat_up * a.group) * 4;
  if (stat_row < kStep) stat[0][kStepPos][stat_row] = stat[1][kStepPos][stat_row] = static_cast<float>(stat_up);
  const int stat_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  auto fetch = [&](int n, int buf) {
    const int tok = first + (steps.parts > 1 ? n / steps.parts : n * steps.tokens);
    const int head = steps.parts > 1 ? n % steps.parts * kStep : 0;
    const int count = min(min(steps.tokens, qs.len - tok) * a.group - head, kStep);
    ql.load(lds + buf * kTile, tok, head, count);
    ol.load(lds + (2 + buf) * kTile, tok, head, count);
    if (stat_wave < kStatRows / kWave) {
      const int64_t at = (qs.start + tok) * a.hq + kvh * a.group + head;
      const uint32_t off = stat_row < count ? stat_off : 0x80000000u;
#pragma unroll
      for (int k = 0; k < kStats; ++k)
        load_words(a.stat + k * a.q_rows * a.hq + at, off, stat[buf][k] + stat_wave * kWave);
    }
  };

  if (n_steps > 0) {  // a step needs a key: j0 < ks.len
    TileLoader<T, HD, C::KEYS, C::W> kl;
    kl.init(a.k.p, ks.start, a.k.row, kvh * a.k.head, a.d, ks.len);
    kl.load(key_tile, j0);
    if (C::VALUES_IN_LDS) {
      kl.init(a.v.p, ks.start, a.v.row, kvh * a.v.head, a.d, ks.len);
      kl.load(val_tile, j0);
    }
    fetch(0, 0);
  }
  for (int n = 0; n < n_steps; ++n) {
    const int buf = n & 1;
    wait_tiles();  // this step's rows are there, the other step's have been read
    if (n + 1 < n_steps) fetch(n + 1, buf ^ 1);
    const int tok = first + (steps.parts > 1 ? n / steps.parts : n * steps.tokens);
    const int last_tok = min(tok + steps.tokens, qs.len) - 1;
    const int least = key_limit(tok, qs.len, ks.len, a.causal, prefix);
    const int most = key_limit(last_tok, qs.len, ks.len, a.causal, prefix);
    const bool masked = min(jw + 32, ks.len) > least;
    const char* qt = lds + buf * kTile;
    const char* dt = lds + (2 + buf) * kTile;
    // wave-uniform: some row of the step sees the wave's keys
    if (jw < most)
#pragma unroll
    for (int part = 0; part < kStep / 32 / C::RW; ++part) {
      const int rb = part * C::RW + rw;  // 32 rows of the step
      f32x16 sc = {}, dp = {};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F f, g;
        row_frag<HD>(qt, rb * 32 + col, t * 16 + half * 8, f);
        row_frag<HD>(key_tile, kw * 32 + col, t * 16 + half * 8, g);
        sc = mma(f, g, sc);
      }
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F f;
        row_frag<HD>(dt, rb * 32 + col, t * 16 + half * 8, f);
        if (C::VALUES_IN_LDS) row_frag<HD>(val_tile, kw * 32 + col, t * 16 + half * 8, vf[0]);
        dp = mma(f, vf[C::VALUES_IN_LDS ? 0 : t], dp);
      }
      // registers 4 g .. 4 g + 3 are rows r, r + 1, r + 2, r + 3
      float p[16], ds[16], sv[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[i] = sc[i];
      const int r = rb * 32 + half * 4;
      float c = scale2;
      if (a.cap > 0.0f) {
        c = cap2;
        tanh_scores<T>(sv, inv_cap);
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] = 1.0f - sv[i] * sv[i];
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 lse = four(stat[buf][kStatLse], r + g * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) p[4 * g + e] = sv[4 * g + e] * c + lse[e];
      }
      if (a.slopes) {
        const float key = static_cast<float>(j - (tok + ks.len - qs.len));
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 pos = four(stat[buf][kStepPos], r + g * 8), slope = four(stat[buf][kStatSlope], r + g * 8);
#pragma unroll
          for (int e = 0; e < 4; ++e) p[4 * g + e] -= slope[e] * fabsf(key - pos[e]);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = exp2_hw(p[i]);
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int pos = __float_as_int(stat[buf][kStatPos][r + (i >> 2) * 8 + (i & 3)]);
          p[i] = j <= pos || j < see_all ? p[i] : 0.0f;
        }
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 delta = four(stat[buf][kStatDelta], r + g * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * g + e] = p[4 * g + e] * (dp[4 * g + e] - delta[e]);
      }
      if (a.cap > 0.0f) {
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] *= dp[i];
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] = dp[i];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const F pf = to_frag<T>(p, t), df = to_frag<T>(ds, t);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          F f;
          col_frag<HD>(dt, rb * 32 + t * 16, i * 32, lane, f);
          dv[i] = mma(f, pf, dv[i]);
          col_frag<HD>(qt, rb * 32 + t * 16, i * 32, lane, f);
          dk[i] = mma(f, df, dk[i]);
        }
      }
    }
  }

  __syncthreads();  // the tiles have been read
  if (C::RW > 1) {
    // the row parts' gradients, added to the first part's in order
    constexpr int kPart = DT * 16 * kWave * sizeof(float);
    static_assert(sizeof(lds) >= C::KW * kPart, "a part of every key wave fits");
    f32x4* mine = reinterpret_cast<f32x4*>(lds + kw * kPart) + lane;
#pragma unroll
    for (int part = 1; part < C::RW; ++part) {
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        f32x16(&g)[DT] = which ? dv : dk;
        if (rw == part)
#pragma unroll
          for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              mine[(i * 4 + e) * kWave] = f32x4{g[i][4 * e], g[i][4 * e + 1], g[i][4 * e + 2], g[i][4 * e + 3]};
        __syncthreads();
        if (rw == 0)
#pragma unroll
          for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const f32x4 x = mine[(i * 4 + e) * kWave];
#pragma unroll
              for (int q = 0; q < 4; ++q) g[i][4 * e + q] += x[q];
            }
        __syncthreads();
      }
    }
    if (rw > 0) return;
  }
  typedef RowWriter<T, HD> S;
  constexpr int kShare = sizeof(lds) / C::KW / 16 * 16;
  static_assert(S::kBytes <= kShare, "a wave's rows fit its share of the tiles");
  char* mine = lds + kw * kShare;
  auto at = [&](void* base, int i) -> T* {
    if (jw + i >= out_rows) return nullptr;
    return static_cast<T*>(base) + ((ks.start + jw + i) * a.hkv + kvh) * a.d;
  };
  S::put(mine, lane, [&](int i, int e) { return live ? dk[i][e] * a.scale : 0.0f; });  // padding: 0
  S::flush(mine, lane, a.d, [&](int i) { return at(a.dk, i); });
  S::put(mine, lane, [&](int i, int e) { return live ? dv[i][e] : 0.0f; });
  S::flush(mine, lane, a.d, [&](int i) { return at(a.dv, i); });
}

// Sum over the lane's part of a row of x y (eight elements).
__device__ inline float dot8(const bf16x8& x, const bf16x8& y) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += static_cast<float>(x[e]) * static_cast<float>(y[e]);
  return s;
}
__device__ inline float dot8(const f32x8s& x, const f32x8s& y) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += x.v[e] * y.v[e];
  return s;
}

// dq of a row tile, what k_attn_dkdv needs of its rows, and its sum of the
// slopes' gradient per head.
//
// delta, in bf16, is taken from the output and what its rounding left: where
// few keys matter, delta is of dP's size and the output's rounding alone would
// be the largest error of dq and dk (2.7e-3 of their norm instead of 2.4e-3, on
// sequences of 100 to 1024 keys with distances weighed).
//
// The slopes' gradient is taken per row, with x_j = P (dP - delta) and t = |p -
// j|, as (sum_j x t - (sum_j x) (sum_j P t) / sum_j P) / sum_j P: the sum of x
// is 0 but for delta's own error, which would else be weighed by every
// distance, and the sum of P is 1 but for the rounding of lse.  Without the
// latter and the sums of 16 keys at a time it was off by up to 2.3e-6 of its
// norm, now by 2e-7 to 9e-7 (fp32 matrix products of the same inputs 3e-7 to
// 2.2e-6), for 8% of this kernel's time where slopes are learnt.
template <typename T, int HD>
__global__ __launch_bounds__(kAttnWaves* kWave, (kResidentRowBlocks<T, HD>)) void k_attn_dq(const AttnArgs a) {
  typedef Tile<T, HD> L;
  typedef typename Frag<T>::type F;
  constexpr int KS = HD / 16, DT = HD / 32;
  constexpr int kTile = kAttnStep * L::kRowBytes;
  __shared__ __align__(1024) char lds[4 * kTile];  // keys and values, two steps of each

  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int half = lane >> 5, col = lane & 31;
  const BlockOf blk = block_of(a, true);
  const int kvh = blk.kvh;
  int s;
  int64_t tile;
  if (a.q_pad > 0) {
    const uint32_t per = static_cast<uint32_t>((a.q_pad * a.group + kAttnRows - 1) / kAttnRows);
    s = static_cast<uint32_t>(blk.tile) / per;
    tile = blk.tile - static_cast<int64_t>(s) * per;
  } else {
    s = find_seq(a.q_off, a.seqs, a.group, kAttnRows, blk.tile, tile);
  }
  const SeqSpan qs = seq_span(a.q_off, s, a.q_pad, a.q_rows), ks = seq_span(a.kv_off, s, a.kv_pad, a.kv_rows);
  const int rows = qs.len * a.group;
  const int64_t out_rows = a.q_pad > 0 ? a.q_pad * a.group : rows;
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;

  // int arithmetic below is for tiles inside the sequence; another tile has no row
  const bool none = tile < 0 || tile * kAttnRows >= out_rows;
  const int r0 = none ? 0 : static_cast<int>(tile) * kAttnRows;
  const int r = r0 + wave * 32 + col;
  const RowOf me = row_of(r, kvh, a.group);
  const bool live = !none && r < rows;
  const int64_t row = (qs.start + me.token) * a.hq + me.head;
  const int limit = live ? key_limit(me.token, qs.len, ks.len, a.causal, prefix) : 0;
  const int last = min(r0 + kAttnRows, rows) - 1;
  const int end = !none && last >= r0 ? key_limit(div_group(last, a.group), qs.len, ks.len, a.causal, prefix) : 0;
  const int w0 = r0 + wave * 32, w1 = min(w0 + 32, rows) - 1;
  const int wave_least = w0 < rows ? key_limit(div_group(w0, a.group), qs.len, ks.len, a.causal, prefix) : 0;
  const int wave_most = w1 >= w0 ? key_limit(div_group(w1, a.group), qs.len, ks.len, a.causal, prefix) : 0;

  TileLoader<T, HD> kl, vl;
  kl.init(a.k.p, ks.start, a.k.row, kvh * a.k.head, a.d, ks.len);
  vl.init(a.v.p, ks.start, a.v.row, kvh * a.v.head, a.d, ks.len);
  if (end > 0) {
    kl.load(lds, 0);
    vl.load(lds + 2 * kTile, 0);
  }
  F qf[KS], of[KS];
  float delta = 0.0f;
  {
    const T* q = static_cast<const T*>(a.q.p) + (qs.start + me.token) * a.q.row + me.head * a.q.head;
    const T* go = static_cast<const T*>(a.dout) + row * a.d;
    const T* o = static_cast<const T*>(a.o) + row * a.d;
    const T* rest = static_cast<const T*>(a.o_rest) + row * a.d;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int k0 = t * 16 + half * 8;
      qf[t] = zero_frag<T>();
      of[t] = zero_frag<T>();
      if (live && k0 < a.d) {
        F x;
        load_frag(q + k0, qf[t]);
        load_frag(go + k0, of[t]);
        load_frag(o + k0, x);
        delta += dot8(x, of[t]);
        if (sizeof(T) == 2 && a.o_rest) {
          load_frag(rest + k0, x);
          delta += dot8(x, of[t]);
        }
      }
    }
    delta = other_half_sum(delta);
  }
  float lse = live ? a.lse_in[row] * kLog2e : INFINITY;
  if (lse == -INFINITY) {  // no key seen: P is 0
    lse = INFINITY;
    delta = 0.0f;
  }
  const int pos = me.token + ks.len - qs.len;
  const int wave_pos0 = div_group(w0, a.group) + ks.len - qs.len;
  const int wave_pos1 = div_group(max(w1, w0), a.group) + ks.len - qs.len;
  const float slope = a.slopes && live ? a.slopes[me.head] * kLog2e : 0.0f;
  if (live && half == 0) {
    const int64_t n = a.q_rows * a.hq;
    a.stat[kStatLse * n + row] = -lse;
    a.stat[kStatDelta * n + row] = delta;
    a.stat[kStatPos * n + row] = __int_as_float(pos);
    a.stat[kStatSlope * n + row] = slope;
  }
  const float scale2 = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap2 = a.cap * kLog2e;

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x16{};
  float sum_p = 0.0f, sum_pt = 0.0f, sum_x = 0.0f, sum_xt = 0.0f;

  int buf = 0;
  for (int j0 = 0; j0 < end; j0 += kAttnStep, buf ^= 1) {
    wait_tiles();
    if (j0 + kAttnStep < end) {
      kl.load(lds + (buf ^ 1) * kTile, j0 + kAttnStep);
      vl.load(lds + (2 + (buf ^ 1)) * kTile, j0 + kAttnStep);
    }
    if (j0 >= wave_most) continue;  // wave-uniform
    const bool masked = j0 + kAttnStep > wave_least;
    const int sign = dist_sign(j0, j0 + kAttnStep - 1, wave_pos0, wave_pos1);
    const char* kt = lds + buf * kTile;
    const char* vt = lds + (2 + buf) * kTile;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 sc = {}, dp = {};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F f;
        row_frag<HD>(kt, kb * 32 + col, t * 16 + half * 8, f);
        sc = mma(f, qf[t], sc);
      }
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F f;
        row_frag<HD>(vt, kb * 32 + col, t * 16 + half * 8, f);
        dp = mma(f, of[t], dp);
      }
      const int j = j0 + kb * 32 + half * 4;  // register i is key j + (i / 4) * 8 + i % 4
      const float dist = static_cast<float>(j - pos);
      float p[16], ds[16], sv[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[i] = sc[i];
      float c = scale2;
      if (a.cap > 0.0f) {
        c = cap2;
        tanh_scores<T>(sv, inv_cap);
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] = 1.0f - sv[i] * sv[i];
      }
      if (!a.slopes) {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = sv[i] * c - lse;
      } else if (sign != 0) {
        const float e = sign > 0 ? slope : -slope, b = dist * e - lse;
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = sv[i] * c + (e * static_cast<float>((i >> 2) * 8 + (i & 3)) + b);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          p[i] = sv[i] * c - (slope * fabsf(dist + static_cast<float>((i >> 2) * 8 + (i & 3))) + lse);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = exp2_hw(p[i]);
      if (masked) {
        const int left = limit - j;
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = (i >> 2) * 8 + (i & 3) < left ? p[i] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] = p[i] * (dp[i] - delta);
      if (a.slope_part) {  // the 16 keys' sums first: shorter chains, less rounding
        float sp = 0.0f, x = 0.0f, pt = 0.0f, xt = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sp += p[i];
          x += dp[i];
        }
        if (sign != 0) {  // one side of the row: |dist + c| = -sign (dist + c)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float c = static_cast<float>((i >> 2) * 8 + (i & 3));
            pt += p[i] * c;
            xt += dp[i] * c;
          }
          const float e = sign > 0 ? -1.0f : 1.0f;
          pt = e * (dist * sp + pt);
          xt = e * (dist * x + xt);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float t = fabsf(dist + static_cast<float>((i >> 2) * 8 + (i & 3)));
            pt += p[i] * t;
            xt += dp[i] * t;
          }
        }
        sum_p += sp;
        sum_x += x;
        sum_pt += pt;
        sum_xt += xt;
      }
      if (a.cap > 0.0f) {
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] *= dp[i];
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] = dp[i];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const F df = to_frag<T>(ds, t);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          F f;
          col_frag<HD>(kt, kb * 32 + t * 16, i * 32, lane, f);
          acc[i] = mma(f, df, acc[i]);
        }
      }
    }
  }

  typedef RowWriter<T, HD> S;
  static_assert(S::kBytes <= kTile, "a wave's rows fit its share of the tiles");
  __syncthreads();  // the tiles have been read
  if (!none) {
    char* mine = lds + wave * kTile;
    S::put(mine, lane, [&](int i, int e) { return live ? acc[i][e] * a.scale : 0.0f; });  // padding: 0
    S::flush(mine, lane, a.d, [&](int i) -> T* {
      if (w0 + i >= out_rows) return nullptr;
      const RowOf x = row_of(w0 + i, kvh, a.group);
      return static_cast<T*>(a.dq) + ((qs.start + x.token) * a.hq + x.head) * a.d;
    });
  }
  if (a.slope_part) {
    __syncthreads();  // the rows have been read
    float* per_row = reinterpret_cast<float*>(lds);
    const float sp = other_half_sum(sum_p), pt = other_half_sum(sum_pt), sx = other_half_sum(sum_x), sxt = other_half_sum(sum_xt);
    if (half == 0) per_row[wave * 32 + col] = live && sp != 0.0f ? (sx * (pt / sp) - sxt) / sp : 0.0f;
    __syncthreads();
    // rows of one head are `group` apart; every block's first row is head r0 % group
    for (int g = threadIdx.x; g < a.group; g += kAttnWaves * kWave) {
      float sum = 0.0f;
      for (int i = (g - r0 % a.group + a.group) % a.group; i < kAttnRows; i += a.group) sum += per_row[i];
      a.slope_part[blk.tile * a.hq + kvh * a.group + g] = sum;
    }
  }
}

// Adds up the row tiles' parts of the slopes' gradient, a block per head.
constexpr int kSlopeThreads = 1024;
__global__ __launch_bounds__(kSlopeThreads) void k_attn_dslopes(const AttnArgs a, int64_t tiles) {
  __shared__ double sh[kSlopeThreads];
  double s = 0.0;
#pragma unroll 8
  for (int64_t t = threadIdx.x; t < tiles; t += kSlopeThreads) s += a.slope_part[t * a.hq + blockIdx.x];
  sh[threadIdx.x] = s;
  for (int w = kSlopeThreads / 2; w > 0; w >>= 1) {
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < w) sh[threadIdx.x] += sh[threadIdx.x + w];
  }
  if (threadIdx.x == 0) a.dslopes[blockIdx.x] = static_cast<float>(sh[0]);
}

int64_t key_tiles(const AttnArgs& a, int keys) {
  if (a.seqs == 0) return 0;
  if (a.kv_pad > 0) return a.seqs * ((a.kv_pad + keys - 1) / keys);
  return a.kv_rows / keys + a.seqs;
}

template <typename T, int HD, bool FEW>
void run_keys(const AttnArgs& a, hipStream_t s) {
  typedef KeyShape<T, HD, FEW> C;
  launch_blocks<C::W * kWave>(k_attn_dkdv<T, HD, FEW>, a, key_tiles(a, C::KEYS) * a.hkv, s);
}

// Where the larger tiles make fewer blocks than this, two to three times what the
// GPU runs at once, the longest of them bounds the pass, and the small shape is
// taken.  dk and dv with small / large tiles, us: 128 bf16, 128 large tiles (one
// sequence of 8000, two heads) 233 / 572, 660 (24 documents, four query heads a
// key head) 542 / 668, 2256 (32 sequences, eight heads) 524 / 435; 64 bf16, 314
// (eight query heads a key head) 162 / 295, 1410 110 / 117, 24576 1238 / 938; 32
// fp32, 128 lists 114 / 137.
constexpr int64_t kFewKeyBlocks = 1536;

template <typename T, int HD>
hipError_t run(const AttnArgs& a, hipStream_t s) {
  const int64_t qt = attn_row_tiles(a);
  launch_blocks<kAttnWaves * kWave>(k_attn_dq<T, HD>, a, qt * a.hkv, s);
  bool few = false;
  if constexpr (HD * sizeof(T) <= 256) {
    few = key_tiles(a, KeyShape<T, HD, false>::KEYS) * a.hkv < kFewKeyBlocks;
    if (few) run_keys<T, HD, true>(a, s);
  }
  if (!few) run_keys<T, HD, false>(a, s);
  if (a.dslopes) k_attn_dslopes<<<a.hq, kSlopeThreads, 0, s>>>(a, qt);
  return hipGetLastError();
}

template <typename T>
hipError_t run_type(const AttnArgs& a, hipStream_t s) {
  if (a.d <= 32) return run<T, 32>(a, s);
  if (a.d <= 64) return run<T, 64>(a, s);
  return run<T, 128>(a, s);
}

}  // namespace

hipError_t launch_attn_bwd(const AttnArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? run_type<uint16_t>(a, s) : run_type<float>(a, s);
}

}  // namespace rs
