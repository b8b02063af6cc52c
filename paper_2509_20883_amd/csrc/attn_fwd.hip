// Attention over ragged sequences, forward (gfx950).
//
//   s_ij = cap(scale q_i.k_j) - slope_h |p_i - j|, p_i = i + Lk - Lq
//   out_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp(s_ij)
//
// over the keys of the query's sequence that it sees.  One pass over the keys
// with the running maximum and sum of the softmax (Milakov & Gimelshein 2018),
// in base 2.  A block takes 128 packed rows (tokens times the query heads of
// one key head) and walks over the keys 64 at a time; a wave owns 32 rows, one
// per lane column: its maximum, sum and rescaling are the lane's own scalars.
#include <hip/hip_runtime.h>

#include "attn_common.h"

#pragma clang fp contract(fast)

namespace rs {
namespace {

template <typename T, int HD>
__global__ __launch_bounds__(kAttnWaves* kWave) void k_attn_fwd(const AttnArgs a) {
  typedef Tile<T, HD> L;
  typedef typename Frag<T>::type F;
  constexpr int KS = HD / 16;  // product steps over d
  constexpr int DT = HD / 32;  // 32-column tiles of the output
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
  const int rows = qs.len * a.group;  // with a key: the others are padding
  const int64_t out_rows = a.q_pad > 0 ? a.q_pad * a.group : rows;
  if (tile * kAttnRows >= out_rows) return;  // block-uniform
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;

  const int r0 = static_cast<int>(tile) * kAttnRows;
  const int r = r0 + wave * 32 + col;  // the lane's row
  const RowOf me = row_of(r, kvh, a.group);
  const bool live = r < rows;
  const int limit = live ? key_limit(me.token, qs.len, ks.len, a.causal, prefix) : 0;
  // limits do not fall along the rows: the block's last row sees the most keys
  const int last = min(r0 + kAttnRows, rows) - 1;
  const int block_limit = last >= r0 ? key_limit(last / a.group, qs.len, ks.len, a.causal, prefix) : 0;

  F qf[KS];
  {
    const T* q = static_cast<const T*>(a.q.p) + (qs.start + me.token) * a.q.row + me.head * a.q.head;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int k0 = t * 16 + half * 8;
      qf[t] = zero_frag<T>();
      if (live && k0 < a.d) load_frag(q + k0, qf[t]);
    }
  }
  const float pos = static_cast<float>(me.token + ks.len - qs.len);
  const float slope = a.slopes && live ? a.slopes[me.head] * kLog2e : 0.0f;
  const float c = a.scale * kLog2e, inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap2 = a.cap * kLog2e;

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x16{};
  float m = -INFINITY, l = 0.0f;

  const T* kp = static_cast<const T*>(a.k.p) + ks.start * a.k.row + kvh * a.k.head;
  const T* vp = static_cast<const T*>(a.v.p) + ks.start * a.v.row + kvh * a.v.head;
  for (int j0 = 0; j0 < block_limit; j0 += kAttnStep) {
    __syncthreads();  // the previous step's tiles have been read
    stage<T, HD, kAttnStep>(kt, a.d, [&](int i) { return j0 + i < ks.len ? kp + (j0 + i) * a.k.row : nullptr; });
    stage<T, HD, kAttnStep>(vt, a.d, [&](int i) { return j0 + i < ks.len ? vp + (j0 + i) * a.v.row : nullptr; });
    __syncthreads();

    float p[2][16];
    float top = m;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 sc = {};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F kf;
        row_frag<HD>(kt, kb * 32 + col, t * 16 + half * 8, kf);
        sc = mma(kf, qf[t], sc);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = j0 + kb * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
        float x = a.cap > 0.0f ? cap2 * tanh_of<T>(sc[i] * inv_cap) : sc[i] * c;
        if (a.slopes) x -= slope * fabsf(static_cast<float>(j) - pos);
        x = j < limit ? x : -INFINITY;
        p[kb][i] = x;
        top = fmaxf(top, x);
      }
    }
    top = other_half_max(top);
    const float base = top == -INFINITY ? 0.0f : top;  // no key seen yet
    const float alpha = exp2_hw(m - base);
    m = top;
    float sum = 0.0f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[kb][i] = exp2_hw(p[kb][i] - base);
        sum += p[kb][i];
      }
    l = l * alpha + sum;  // this half's keys
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] *= alpha;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const F pf = to_frag<T>(p[kb], t);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          F vf;
          col_frag<HD>(vt, kb * 32 + t * 16, i * 32, lane, vf);
          acc[i] = mma(vf, pf, acc[i]);
        }
      }
  }

  if (r >= out_rows) return;
  l = other_half_sum(l);
  const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);  // no key: 0; NaN stays
  const int64_t row = (qs.start + me.token) * a.hq + me.head;
  T* out = static_cast<T*>(a.out) + row * a.d;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d0 = i * 32 + g * 8 + half * 4;
      if (d0 >= a.d) continue;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = acc[i][4 * g + e] * inv;
      store4(out + d0, x[0], x[1], x[2], x[3]);
      if (sizeof(T) == 2 && a.rest)
        store4(static_cast<uint16_t*>(a.rest) + row * a.d + d0, rest_bf16(x[0]), rest_bf16(x[1]), rest_bf16(x[2]),
               rest_bf16(x[3]));
    }
  if (a.lse && half == 0) a.lse[row] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
}

template <typename T, int HD>
hipError_t run(const AttnArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(attn_row_tiles(a)), a.hkv);
  const size_t lds = 2 * kAttnStep * Tile<T, HD>::kRowBytes;
  k_attn_fwd<T, HD><<<grid, kAttnWaves * kWave, lds, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t run_type(const AttnArgs& a, hipStream_t s) {
  if (a.d <= 32) return run<T, 32>(a, s);
  if (a.d <= 64) return run<T, 64>(a, s);
  return run<T, 128>(a, s);
}

}  // namespace

int64_t attn_row_tiles(const AttnArgs& a) {
  if (a.seqs == 0) return 0;
  if (a.q_pad > 0) return a.seqs * ((a.q_pad * a.group + kAttnRows - 1) / kAttnRows);
  return a.q_rows * a.group / kAttnRows + a.seqs;
}

hipError_t launch_attn_fwd(const AttnArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? run_type<uint16_t>(a, s) : run_type<float>(a, s);
}

}  // namespace rs
