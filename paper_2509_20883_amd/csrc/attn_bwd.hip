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
// add up in registers), one over row tiles for dq, walking over the keys.
#include <hip/hip_runtime.h>

#include "attn_common.h"

#pragma clang fp contract(fast)

namespace rs {
namespace {

// delta of every row, a wave per row (0 where the row is padding).  In bf16
// it is taken from the output and what its rounding left: where few keys
// matter, delta is of dP's size and the output's rounding alone would be the
// largest error of dq and dk (2.7e-3 of their norm instead of 2.4e-3, on
// sequences of 100 to 1024 keys with distances weighed).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_attn_delta(const AttnArgs a) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t n = a.q_rows * a.hq;
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * (kBlock / kWave) + threadIdx.x / kWave; r < n;
       r += static_cast<int64_t>(gridDim.x) * (kBlock / kWave)) {
    float s = 0.0f;
    if (a.lse_in[r] != -INFINITY)  // a row without keys, or past its sequence's end, is not read
      for (int i = lane; i < a.d; i += kWave) {
        const T x = static_cast<const T*>(a.o)[r * a.d + i], y = static_cast<const T*>(a.dout)[r * a.d + i];
        if (sizeof(T) == 2) {
          float o = bf16_to_f32(static_cast<uint16_t>(x));
          if (a.o_rest) o += bf16_to_f32(static_cast<const uint16_t*>(a.o_rest)[r * a.d + i]);
          s += o * bf16_to_f32(static_cast<uint16_t>(y));
        } else s += static_cast<float>(x) * static_cast<float>(y);
      }
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) s += __shfl_xor(s, d, kWave);
    if (lane == 0) a.delta[r] = s;
  }
}

// Capped score in base 2 (and, for the gradient, the cap's derivative).
template <typename T>
__device__ inline float score2(float dot, float c, float inv_cap, float cap2, float& deriv) {
  if (cap2 > 0.0f) {
    const float th = tanh_of<T>(dot * inv_cap);
    deriv = 1.0f - th * th;
    return cap2 * th;
  }
  deriv = 1.0f;
  return dot * c;
}

template <typename T, int HD>
__global__ __launch_bounds__(kAttnWaves* kWave) void k_attn_dkdv(const AttnArgs a) {
  typedef Tile<T, HD> L;
  typedef typename Frag<T>::type F;
  constexpr int KS = HD / 16, DT = HD / 32;
  extern __shared__ __align__(16) char lds[];
  char* qt = lds;
  char* dt = lds + kAttnStep * L::kRowBytes;
  float* row_lse = reinterpret_cast<float*>(lds + 2 * kAttnStep * L::kRowBytes);  // base 2, +inf: no key seen
  float* row_delta = row_lse + kAttnStep;
  float* row_pos = row_delta + kAttnStep;
  float* row_slope = row_pos + kAttnStep;
  int* row_limit = reinterpret_cast<int*>(row_slope + kAttnStep);

  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int half = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.y;
  int s;
  int64_t tile;
  if (a.kv_pad > 0) {
    const int64_t per = (a.kv_pad + kAttnRows - 1) / kAttnRows;
    s = static_cast<int>(blockIdx.x / per);
    tile = blockIdx.x - s * per;
  } else {
    s = find_seq(a.kv_off, a.seqs, 1, kAttnRows, blockIdx.x, tile);
  }
  const SeqSpan qs = seq_span(a.q_off, s, a.q_pad, a.q_rows), ks = seq_span(a.kv_off, s, a.kv_pad, a.kv_rows);
  const int64_t out_rows = a.kv_pad > 0 ? a.kv_pad : ks.len;
  if (tile * kAttnRows >= out_rows) return;  // block-uniform
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;
  const int rows = qs.len * a.group;

  const int j0 = static_cast<int>(tile) * kAttnRows;
  const int j = j0 + wave * 32 + col;  // the lane's key
  const bool live = j < ks.len;
  F kf[KS], vf[KS];
  {
    const T* k = static_cast<const T*>(a.k.p) + (ks.start + j) * a.k.row + kvh * a.k.head;
    const T* v = static_cast<const T*>(a.v.p) + (ks.start + j) * a.v.row + kvh * a.v.head;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int k0 = t * 16 + half * 8;
      kf[t] = zero_frag<T>();
      vf[t] = zero_frag<T>();
      if (live && k0 < a.d) {
        load_frag(k + k0, kf[t]);
        load_frag(v + k0, vf[t]);
      }
    }
  }
  const float c = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap2 = a.cap * kLog2e;
  const float key = static_cast<float>(j);

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
  for (int r0 = first * a.group; r0 < rows; r0 += kAttnStep) {
    __syncthreads();
    auto addr = [&](const void* base, int64_t row, int64_t head, int i) -> const T* {
      if (r0 + i >= rows) return nullptr;
      const RowOf x = row_of(r0 + i, kvh, a.group);
      return static_cast<const T*>(base) + (qs.start + x.token) * row + x.head * head;
    };
    stage<T, HD, kAttnStep>(qt, a.d, [&](int i) { return addr(a.q.p, a.q.row, a.q.head, i); });
    stage<T, HD, kAttnStep>(dt, a.d, [&](int i) { return addr(a.dout, int64_t(a.hq) * a.d, a.d, i); });
    if (threadIdx.x < kAttnStep) {
      const int i = threadIdx.x, r = r0 + i;
      float lse = INFINITY, delta = 0.0f, slope = 0.0f, pos = 0.0f;
      int limit = 0;
      if (r < rows) {
        const RowOf x = row_of(r, kvh, a.group);
        const int64_t at = (qs.start + x.token) * a.hq + x.head;
        lse = a.lse_in[at] * kLog2e;
        if (lse == -INFINITY) lse = INFINITY;
        delta = a.delta[at];
        pos = static_cast<float>(x.token + ks.len - qs.len);
        limit = key_limit(x.token, qs.len, ks.len, a.causal, prefix);
        if (a.slopes) slope = a.slopes[x.head] * kLog2e;
      }
      row_lse[i] = lse;
      row_delta[i] = delta;
      row_pos[i] = pos;
      row_slope[i] = slope;
      row_limit[i] = limit;
    }
    __syncthreads();

#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      f32x16 sc = {}, dp = {};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F f;
        row_frag<HD>(qt, rb * 32 + col, t * 16 + half * 8, f);
        sc = mma(f, kf[t], sc);
      }
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F f;
        row_frag<HD>(dt, rb * 32 + col, t * 16 + half * 8, f);
        dp = mma(f, vf[t], dp);
      }
      float p[16], ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = rb * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
        float deriv;
        float x = score2<T>(sc[i], c, inv_cap, cap2, deriv);
        if (a.slopes) x -= row_slope[r] * fabsf(key - row_pos[r]);
        const bool sees = j < row_limit[r];
        p[i] = sees ? exp2_hw(x - row_lse[r]) : 0.0f;
        ds[i] = sees ? p[i] * (dp[i] - row_delta[r]) * deriv : 0.0f;
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

  if (j >= out_rows) return;
  const int64_t row = (ks.start + j) * a.hkv + kvh;
  T* dkp = static_cast<T*>(a.dk) + row * a.d;
  T* dvp = static_cast<T*>(a.dv) + row * a.d;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d0 = i * 32 + g * 8 + half * 4;
      if (d0 < a.d) {
        store4(dkp + d0, dk[i][4 * g] * a.scale, dk[i][4 * g + 1] * a.scale, dk[i][4 * g + 2] * a.scale,
               dk[i][4 * g + 3] * a.scale);
        store4(dvp + d0, dv[i][4 * g], dv[i][4 * g + 1], dv[i][4 * g + 2], dv[i][4 * g + 3]);
      }
    }
}

// dq of a row tile, and its sum of the slopes' gradient per head.  The latter
// is taken per row as sum_j P dP t - (sum_j P dP)(sum_j P t), t = |p - j|, all
// fp32 from this pass's own P and dP: delta comes from the rounded output and
// would carry its error into a sum that cancels.
template <typename T, int HD>
__global__ __launch_bounds__(kAttnWaves* kWave) void k_attn_dq(const AttnArgs a) {
  typedef Tile<T, HD> L;
  typedef typename Frag<T>::type F;
  constexpr int KS = HD / 16, DT = HD / 32;
  extern __shared__ __align__(16) char lds[];
  char* kt = lds;
  char* vt = lds + kAttnStep * L::kRowBytes;

  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int half = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.y;
  int s;
  int64_t tile;
  if (a.q_pad > 0) {
    const int64_t per = (a.q_pad * a.group + kAttnRows - 1) / kAttnRows;
    s = static_cast<int>(blockIdx.x / per);
    tile = blockIdx.x - s * per;
  } else {
    s = find_seq(a.q_off, a.seqs, a.group, kAttnRows, blockIdx.x, tile);
  }
  const SeqSpan qs = seq_span(a.q_off, s, a.q_pad, a.q_rows), ks = seq_span(a.kv_off, s, a.kv_pad, a.kv_rows);
  const int rows = qs.len * a.group;
  const int64_t out_rows = a.q_pad > 0 ? a.q_pad * a.group : rows;
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;

  // int arithmetic below is for tiles inside the sequence; another tile has no row
  const bool none = tile * kAttnRows >= out_rows;
  const int r0 = none ? 0 : static_cast<int>(tile) * kAttnRows;
  const int r = r0 + wave * 32 + col;
  const RowOf me = row_of(r, kvh, a.group);
  const bool live = !none && r < rows;
  const int64_t row = (qs.start + me.token) * a.hq + me.head;
  const int limit = live ? key_limit(me.token, qs.len, ks.len, a.causal, prefix) : 0;
  const int last = min(r0 + kAttnRows, rows) - 1;
  const int block_limit = !none && last >= r0 ? key_limit(last / a.group, qs.len, ks.len, a.causal, prefix) : 0;

  F qf[KS], of[KS];
  {
    const T* q = static_cast<const T*>(a.q.p) + (qs.start + me.token) * a.q.row + me.head * a.q.head;
    const T* o = static_cast<const T*>(a.dout) + row * a.d;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int k0 = t * 16 + half * 8;
      qf[t] = zero_frag<T>();
      of[t] = zero_frag<T>();
      if (live && k0 < a.d) {
        load_frag(q + k0, qf[t]);
        load_frag(o + k0, of[t]);
      }
    }
  }
  float lse = live ? a.lse_in[row] * kLog2e : INFINITY;
  if (lse == -INFINITY) lse = INFINITY;
  const float delta = live ? a.delta[row] : 0.0f;
  const float pos = static_cast<float>(me.token + ks.len - qs.len);
  const float slope = a.slopes && live ? a.slopes[me.head] * kLog2e : 0.0f;
  const float c = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap2 = a.cap * kLog2e;

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x16{};
  float sum_pt = 0.0f, sum_pd = 0.0f, sum_pdt = 0.0f;

  const T* kp = static_cast<const T*>(a.k.p) + ks.start * a.k.row + kvh * a.k.head;
  const T* vp = static_cast<const T*>(a.v.p) + ks.start * a.v.row + kvh * a.v.head;
  for (int j0 = 0; j0 < block_limit; j0 += kAttnStep) {
    __syncthreads();
    stage<T, HD, kAttnStep>(kt, a.d, [&](int i) { return j0 + i < ks.len ? kp + (j0 + i) * a.k.row : nullptr; });
    stage<T, HD, kAttnStep>(vt, a.d, [&](int i) { return j0 + i < ks.len ? vp + (j0 + i) * a.v.row : nullptr; });
    __syncthreads();
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
      float ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = j0 + kb * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
        float deriv;
        float x = score2<T>(sc[i], c, inv_cap, cap2, deriv);
        const float t = fabsf(static_cast<float>(j) - pos);
        if (a.slopes) x -= slope * t;
        const bool sees = j < limit;
        const float p = sees ? exp2_hw(x - lse) : 0.0f;
        ds[i] = sees ? p * (dp[i] - delta) * deriv : 0.0f;
        if (a.slope_part) {
          const float pd = sees ? p * dp[i] : 0.0f;
          sum_pt += p * t;
          sum_pd += pd;
          sum_pdt += pd * t;
        }
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

  if (!none && r < out_rows) {
    T* dq = static_cast<T*>(a.dq) + row * a.d;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d0 = i * 32 + g * 8 + half * 4;
        if (d0 < a.d)
          store4(dq + d0, acc[i][4 * g] * a.scale, acc[i][4 * g + 1] * a.scale, acc[i][4 * g + 2] * a.scale,
                 acc[i][4 * g + 3] * a.scale);
      }
  }
  if (a.slope_part) {
    __syncthreads();  // the tiles have been read
    float* per_row = reinterpret_cast<float*>(lds);
    const float pt = other_half_sum(sum_pt), pd = other_half_sum(sum_pd), pdt = other_half_sum(sum_pdt);
    if (half == 0) per_row[wave * 32 + col] = live ? pd * pt - pdt : 0.0f;
    __syncthreads();
    // rows of one head are `group` apart; every block's first row is head r0 % group
    for (int g = threadIdx.x; g < a.group; g += kAttnWaves * kWave) {
      float sum = 0.0f;
      for (int i = (g - r0 % a.group + a.group) % a.group; i < kAttnRows; i += a.group) sum += per_row[i];
      a.slope_part[static_cast<int64_t>(blockIdx.x) * a.hq + kvh * a.group + g] = sum;
    }
  }
}

// Adds up the row tiles' parts of the slopes' gradient, a block per head.
__global__ __launch_bounds__(kBlock) void k_attn_dslopes(const AttnArgs a, int64_t tiles) {
  __shared__ double sh[kBlock];
  double s = 0.0;
  for (int64_t t = threadIdx.x; t < tiles; t += kBlock) s += a.slope_part[t * a.hq + blockIdx.x];
  sh[threadIdx.x] = s;
  for (int w = kBlock / 2; w > 0; w >>= 1) {
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < w) sh[threadIdx.x] += sh[threadIdx.x + w];
  }
  if (threadIdx.x == 0) a.dslopes[blockIdx.x] = static_cast<float>(sh[0]);
}

int64_t key_tiles(const AttnArgs& a) {
  if (a.seqs == 0) return 0;
  if (a.kv_pad > 0) return a.seqs * ((a.kv_pad + kAttnRows - 1) / kAttnRows);
  return a.kv_rows / kAttnRows + a.seqs;
}

template <typename T, int HD>
hipError_t run(const AttnArgs& a, hipStream_t s) {
  const size_t lds = 2 * kAttnStep * Tile<T, HD>::kRowBytes;
  const dim3 kg(static_cast<unsigned>(key_tiles(a)), a.hkv), qg(static_cast<unsigned>(attn_row_tiles(a)), a.hkv);
  if (a.q_rows > 0) k_attn_delta<T><<<grid_for(a.q_rows * a.hq, kBlock / kWave, 1 << 16), kBlock, 0, s>>>(a);
  if (kg.x > 0) k_attn_dkdv<T, HD><<<kg, kAttnWaves * kWave, lds + 5 * 4 * kAttnStep, s>>>(a);
  if (qg.x > 0) k_attn_dq<T, HD><<<qg, kAttnWaves * kWave, lds, s>>>(a);
  if (a.dslopes) k_attn_dslopes<<<a.hq, kBlock, 0, s>>>(a, qg.x);
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
