// Layer norm over the last axis, forward and backward (gfx950).
//
//   mean = sum x / D, var = sum (x - mean)^2 / D, rstd = 1 / sqrt(var + eps)
//   xhat = (x - mean) rstd,  y = xhat w + b
//   g = dy w,  dx = rstd (g - mean_D(g) - xhat mean_D(g xhat))
//   dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// A handful of operations per element, so memory bounds every size: the
// floor is one read of x (and dy) and one write of y (dx).  Statistics,
// sums and gradients are fp32; only y, dx, dw and db are rounded, once.
// The variance is the mean square about the mean, not E[x^2] - mean^2, which
// cancels for rows far from zero.  Rows whose mask byte is 0 are never read:
// their y and dx are 0 and they add nothing to dw and db.
//
// 65536 rows of 1024 bf16: forward 43 us (6.2 TB/s), backward 67 (6.0) and the
// sums over rows 6; 1,572,864 rows of 128 bf16, 45% of them masked, 134 and 173
// us (4.6 and 4.9 TB/s of the live rows read and all rows written; all rows live
// 148 and 227, 5.4 TB/s, all masked 77, at the rate of plain writes).
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "seq_internal.h"

#pragma clang fp contract(fast)

namespace rs {
namespace {

template <typename T>
__device__ inline float to_f32(T v);
template <>
__device__ inline float to_f32<float>(float v) {
  return v;
}
template <>
__device__ inline float to_f32<uint16_t>(uint16_t v) {
  return bf16_to_f32(v);
}
template <typename T>
__device__ inline T from_f32(float v);
template <>
__device__ inline float from_f32<float>(float v) {
  return v;
}
template <>
__device__ inline uint16_t from_f32<uint16_t>(float v) {
  return f32_to_bf16(v);
}

// Two floats to bf16 (round to nearest even), in one word.
__device__ inline uint32_t pack2_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Weights and their gradients come in either type; a null weight is 1.
__device__ inline float param(const void* p, bool bf16, int64_t i) {
  return bf16 ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

__device__ inline float wave_sum_f(float v) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d >>= 1) v += __shfl_xor(v, d, kWave);
  return v;
}

// The sum over the block, in every thread; `sh` holds one float per wave.
__device__ inline float block_sum_f(float v, float* sh) {
  v = wave_sum_f(v);
  __syncthreads();  // the previous sum has been read
  if ((threadIdx.x & (kWave - 1)) == 0) sh[threadIdx.x / kWave] = v;
  __syncthreads();
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < kBlock / kWave; ++i) t += sh[i];
  return t;
}

// Rows above 8192 elements: a block per row that passes over it three times
// (mean, variance, result); after the first the row comes from the caches.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_ln_fwd_any(const NormArgs a) {
  __shared__ float sh[kBlock / kWave];
  const float inv_d = 1.0f / static_cast<float>(a.dim);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    T* y = static_cast<T*>(a.y) + r * a.y_stride;
    if (a.mask && !a.mask[r]) {  // block-uniform
      for (int64_t i = threadIdx.x; i < a.dim; i += kBlock) y[i] = T(0);
      if (threadIdx.x == 0) {
        if (a.mean_out) a.mean_out[r] = 0.0f;
        if (a.rstd_out) a.rstd_out[r] = 0.0f;
      }
      continue;
    }
    const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < a.dim; i += kBlock) s += to_f32(x[i]);
    const float mean = block_sum_f(s, sh) * inv_d;
    float q = 0.0f;
    for (int64_t i = threadIdx.x; i < a.dim; i += kBlock) {
      const float c = to_f32(x[i]) - mean;
      q += c * c;
    }
    const float rstd = rsqrtf(block_sum_f(q, sh) * inv_d + a.eps);
    for (int64_t i = threadIdx.x; i < a.dim; i += kBlock) {
      float v = (to_f32(x[i]) - mean) * rstd;
      if (a.weight) v *= param(a.weight, a.param_bf16, i);
      if (a.bias) v += param(a.bias, a.param_bf16, i);
      y[i] = from_f32<T>(v);
    }
    if (threadIdx.x == 0) {
      if (a.mean_out) a.mean_out[r] = mean;
      if (a.rstd_out) a.rstd_out[r] = rstd;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_ln_dx_any(const NormArgs a) {
  __shared__ float sh[kBlock / kWave];
  const float inv_d = 1.0f / static_cast<float>(a.dim);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    T* dx = static_cast<T*>(a.dx) + r * a.dx_stride;
    if (a.mask && !a.mask[r]) {  // block-uniform
      for (int64_t i = threadIdx.x; i < a.dim; i += kBlock) dx[i] = T(0);
      continue;
    }
    const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + r * a.dy_stride;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sg = 0.0f, sgx = 0.0f;
    for (int64_t i = threadIdx.x; i < a.dim; i += kBlock) {
      float g = to_f32(dy[i]);
      if (a.weight) g *= param(a.weight, a.param_bf16, i);
      sg += g;
      sgx += g * ((to_f32(x[i]) - mean) * rstd);
    }
    const float mg = block_sum_f(sg, sh) * inv_d, mgx = block_sum_f(sgx, sh) * inv_d;
    for (int64_t i = threadIdx.x; i < a.dim; i += kBlock) {
      float g = to_f32(dy[i]);
      if (a.weight) g *= param(a.weight, a.param_bf16, i);
      const float xhat = (to_f32(x[i]) - mean) * rstd;
      dx[i] = from_f32<T>(rstd * (g - mg - xhat * mgx));
    }
  }
}

// dw and db of a range of rows: a thread per column, partial sums to
// part[range][0 .. dim) and part[range][dim .. 2 dim).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_ln_cols_any(const NormArgs a) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
  if (i >= a.dim) return;
  const int64_t per = (a.rows + a.nparts - 1) / a.nparts;
  for (int p = blockIdx.y; p < a.nparts; p += gridDim.y) {
    const int64_t r0 = p * per, r1 = min(r0 + per, a.rows);
    float dw = 0.0f, db = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
      if (a.mask && !a.mask[r]) continue;
      const float g = to_f32(static_cast<const T*>(a.dy)[r * a.dy_stride + i]);
      dw += g * ((to_f32(static_cast<const T*>(a.x)[r * a.x_stride + i]) - a.mean[r]) * a.rstd[r]);
      db += g;
    }
    float* out = a.part + static_cast<int64_t>(p) * 2 * a.dim;
    out[i] = dw;
    out[a.dim + i] = db;
  }
}

// Adds up the partial sums: 16 columns per block, 64 threads per column, in a
// fixed order, so the result does not change from run to run.
constexpr int kFinishCols = 16, kFinishRows = 64;
__global__ __launch_bounds__(kFinishCols* kFinishRows) void k_ln_cols_finish(const NormArgs a) {
  __shared__ float sh[kFinishRows][kFinishCols + 1];
  const int64_t c = static_cast<int64_t>(blockIdx.x) * kFinishCols + threadIdx.x % kFinishCols;
  const int r = threadIdx.x / kFinishCols;
  float s = 0.0f;
  if (c < 2 * a.dim) {
#pragma unroll 8
    for (int p = r; p < a.nparts; p += kFinishRows) s += a.part[static_cast<int64_t>(p) * 2 * a.dim + c];
  }
  sh[r][threadIdx.x % kFinishCols] = s;
  __syncthreads();
  if (r == 0 && c < 2 * a.dim) {
    float t = 0.0f;
#pragma unroll
    for (int k = 0; k < kFinishRows; ++k) t += sh[k][threadIdx.x];
    void* out = c < a.dim ? a.dweight : a.dbias;
    const int64_t i = c < a.dim ? c : c - a.dim;
    if (out) {
      if (a.param_bf16) static_cast<uint16_t*>(out)[i] = f32_to_bf16(t);
      else static_cast<float*>(out)[i] = t;
    }
  }
}

// ---------------------------------------------------------------------------
// rows up to 8192 elements: a row stays in the registers of G lanes
// ---------------------------------------------------------------------------

// Sum over G lanes (a power of two, all of them in one row of the wave), in
// every lane, without LDS: within 16 lanes by data-parallel primitives
// (neighbours, pairs, halves mirrored), then by lane-row swaps.
template <int CTRL>
__device__ inline float dpp_add(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}
template <int G>
__device__ inline float group_sum(float v) {
  if (G >= 2) v = dpp_add<0xB1>(v);    // quad_perm [1, 0, 3, 2]
  if (G >= 4) v = dpp_add<0x4E>(v);    // quad_perm [2, 3, 0, 1]
  if (G >= 8) v = dpp_add<0x141>(v);   // row_half_mirror
  if (G >= 16) v = dpp_add<0x140>(v);  // row_mirror
  if (G >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (G >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// The same over the row's lanes, a whole block where G is kBlock; `sh` is the
// block's, one float per wave and row, not read again before a later barrier.
template <int G, int R>
__device__ inline void row_sums(float (&v)[R], float* sh) {
#pragma unroll
  for (int k = 0; k < R; ++k) v[k] = group_sum<(G < kWave ? G : kWave)>(v[k]);
  if (G > kWave) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < R; ++k) sh[k * (kBlock / kWave) + wave] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < R; ++k) {
      v[k] = 0.0f;
#pragma unroll
      for (int w = 0; w < kBlock / kWave; ++w) v[k] += sh[k * (kBlock / kWave) + w];
    }
  }
}

// A lane's part of a row: NV pieces of VEC consecutive elements, piece i at
// element (i * G + lane) * VEC.  VEC is 16 bytes' worth, or 1 for rows that
// are not 16-byte aligned or not a multiple of it.  The raw words are loaded
// first and widened later, so that no load waits for another.
template <typename T, int VEC>
struct Raw {
  uint4 w;
};
template <>
struct Raw<float, 1> {
  float w;
};
template <>
struct Raw<uint16_t, 1> {
  uint16_t w;
};
template <typename T, int VEC>
__device__ inline void raw_load(const T* p, Raw<T, VEC>& r) {
  if constexpr (VEC == 1) r.w = *p;
  else r.w = *reinterpret_cast<const uint4*>(p);
}
template <typename T, int VEC>
__device__ inline void raw_widen(const Raw<T, VEC>& r, float* v) {
  if constexpr (VEC == 1) {
    v[0] = to_f32<T>(r.w);
  } else {
    float t[VEC];
    widen16<T, VEC>(r.w, t);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = t[e];
  }
}
template <typename T, int VEC, bool STREAM>
__device__ inline void piece_store(T* p, const float* v) {
  if constexpr (VEC == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    nt_u32x4 w;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack2_bf16(v[2 * e], v[2 * e + 1]);
    }
    if constexpr (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<nt_u32x4*>(p));
    else *reinterpret_cast<nt_u32x4*>(p) = w;
  }
}
// Zeros over a row's pieces.
template <typename T, int VEC, int NV, int G, bool STREAM>
__device__ inline void zero_row(T* p, int dim, int lane) {
  const float z[VEC] = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * G + lane) * VEC;
    if (c < dim) piece_store<T, VEC, STREAM>(p + c, z);
  }
}

// The lane's part of weight or bias (`one` where there is none and past dim),
// in 16-byte loads where `vec` says that the pieces are aligned.
template <int VEC, int NV, int G>
__device__ inline void load_param(const void* p, bool bf16, bool vec, int dim, int lane, float one,
                                  float (&w)[NV * VEC]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c0 = (i * G + lane) * VEC;
    float t[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = one;
    if (p && c0 < dim) {
      if (VEC > 1 && vec) {
        if constexpr (VEC > 1) {
          if (bf16) load_vals<uint16_t, VEC>(static_cast<const uint16_t*>(p) + c0, t);
          else load_vals<float, VEC>(static_cast<const float*>(p) + c0, t);
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) t[e] = param(p, bf16, c0 + e);
      }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[i * VEC + e] = t[e];
  }
}

template <typename T, int VEC, int NV, int G, int R, bool STREAM>
__global__ __launch_bounds__(kBlock) void k_ln_fwd(const NormArgs a) {
  constexpr int RB = kBlock / G;  // rows a block holds at once, R times
  __shared__ float sh[2][R * (kBlock / kWave)];
  const int lane = threadIdx.x % G, grp = threadIdx.x / G;
  const int dim = static_cast<int>(a.dim);
  const float inv_d = 1.0f / static_cast<float>(dim);
  float w[NV * VEC], b[NV * VEC];
  load_param<VEC, NV, G>(a.weight, a.param_bf16, a.param16, dim, lane, 1.0f, w);
  load_param<VEC, NV, G>(a.bias, a.param_bf16, a.param16, dim, lane, 0.0f, b);
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * RB * R; r0 < a.rows; r0 += static_cast<int64_t>(gridDim.x) * RB * R) {
    bool in[R], live[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t r = r0 + k * RB + grp;
      in[k] = r < a.rows;
      live[k] = in[k] && (!a.mask || a.mask[r]);
    }
    const T* x0 = static_cast<const T*>(a.x) + (r0 + grp) * a.x_stride;
    T* y0 = static_cast<T*>(a.y) + (r0 + grp) * a.y_stride;
    bool any = false;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (in[k] && !live[k]) {
        zero_row<T, VEC, NV, G, STREAM>(y0 + k * RB * a.y_stride, dim, lane);
        if (lane == 0) {
          if (a.mean_out) a.mean_out[r0 + k * RB + grp] = 0.0f;
          if (a.rstd_out) a.rstd_out[r0 + k * RB + grp] = 0.0f;
        }
      }
      any |= live[k];
    }
    if (!__any(any)) continue;  // padding; G > 64: the whole block agrees
    Raw<T, VEC> raw[R][NV];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const T* x = x0 + k * RB * a.x_stride;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + lane) * VEC;
        raw[k][i] = Raw<T, VEC>{};
        if (live[k] && c < dim) raw_load<T, VEC>(x + c, raw[k][i]);
      }
    }
    float v[R][NV * VEC], mean[R], q[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) raw_widen<T, VEC>(raw[k][i], &v[k][i * VEC]);
#pragma unroll
      for (int i = 0; i < NV * VEC; ++i) mean[k] += v[k][i];
    }
    row_sums<G, R>(mean, sh[0]);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] *= inv_d;
      q[k] = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if ((i * G + lane) * VEC < dim) {  // pieces do not straddle the end
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            v[k][i * VEC + e] -= mean[k];
            q[k] += v[k][i * VEC + e] * v[k][i * VEC + e];
          }
        }
      }
    }
    row_sums<G, R>(q, sh[1]);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (!live[k]) continue;
      const int64_t r = r0 + k * RB + grp;
      const float rstd = rsqrtf(q[k] * inv_d + a.eps);
      T* y = y0 + k * RB * a.y_stride;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + lane) * VEC;
        if (c >= dim) continue;
        float o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = v[k][i * VEC + e] * rstd * w[i * VEC + e] + b[i * VEC + e];
        piece_store<T, VEC, STREAM>(y + c, o);
      }
      if (lane == 0) {
        if (a.mean_out) a.mean_out[r] = mean[k];
        if (a.rstd_out) a.rstd_out[r] = rstd;
      }
    }
  }
}

// dx, and the block's sums of dw and db: a lane keeps the sums of its columns
// over the block's rows in registers, the groups of a wave add theirs by lane
// swaps and the waves through LDS, and one row of `part` is written per block.
template <typename T, int VEC, int NV, int G, int R, bool STREAM>
__global__ __launch_bounds__(kBlock) void k_ln_bwd(const NormArgs a) {
  constexpr int RB = kBlock / G, E = NV * VEC;
  constexpr int kWaves = kBlock / kWave, GW = G < kWave ? G : kWave;
  __shared__ float sh[2][2 * R * kWaves];
  __shared__ float cols[G < kBlock ? kWaves - 1 : 1][GW * E];
  const int lane = threadIdx.x % G, grp = threadIdx.x / G, wave = threadIdx.x / kWave;
  const int dim = static_cast<int>(a.dim);
  const float inv_d = 1.0f / static_cast<float>(dim);
  float w[E], dw[E], db[E];
  load_param<VEC, NV, G>(a.weight, a.param_bf16, a.param16, dim, lane, 1.0f, w);
#pragma unroll
  for (int i = 0; i < E; ++i) dw[i] = db[i] = 0.0f;
  int turn = 0;
  // A row's mask byte, then the row, then its result are one chain of memory
  // trips.  Narrow rows, and those that a block holds in 8 elements a thread, are
  // loaded a turn ahead and their mask bytes two (the padded copy of 1536
  // sequences, 128 bf16: 187 -> 173 us; 20011 rows of 2047 fp32, both directions,
  // 167 -> 155); others have enough loads on their way with the fourth wave per
  // SIMD that this would cost (65536 rows of 1024 bf16: 67 us, a turn ahead 72).
  constexpr bool kAhead = G <= 32 || (G > kWave && E <= 8);
  struct Rows {
    bool in[R], live[R];
    Raw<T, VEC> rx[R][NV], rg[R][NV];
    float mean[R], rstd[R];
  };
  const int64_t step = static_cast<int64_t>(gridDim.x) * RB * R;
  uint8_t bytes[R];
  auto load_bytes = [&](int64_t r0) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t r = r0 + k * RB + grp;
      bytes[k] = r < a.rows ? (a.mask ? a.mask[r] : 1) : 0;
    }
  };
  auto load_rows = [&](int64_t r0, Rows& n) {
    const T* x0 = static_cast<const T*>(a.x) + (r0 + grp) * a.x_stride;
    const T* dy0 = static_cast<const T*>(a.dy) + (r0 + grp) * a.dy_stride;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      n.in[k] = r0 + k * RB + grp < a.rows;
      n.live[k] = bytes[k] != 0;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t r = r0 + k * RB + grp;
      n.mean[k] = n.live[k] ? a.mean[r] : 0.0f;
      n.rstd[k] = n.live[k] ? a.rstd[r] : 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + lane) * VEC;
        n.rx[k][i] = Raw<T, VEC>{};
        n.rg[k][i] = Raw<T, VEC>{};
        if (n.live[k] && c < dim) {
          raw_load<T, VEC>(x0 + k * RB * a.x_stride + c, n.rx[k][i]);
          raw_load<T, VEC>(dy0 + k * RB * a.dy_stride + c, n.rg[k][i]);
        }
      }
    }
  };
  auto work = [&](int64_t r0, Rows& cur) {
    bool(&in)[R] = cur.in;
    bool(&live)[R] = cur.live;
    Raw<T, VEC>(&rx)[R][NV] = cur.rx;
    Raw<T, VEC>(&rg)[R][NV] = cur.rg;
    float(&mean)[R] = cur.mean;
    float(&rstd)[R] = cur.rstd;
    T* dx0 = static_cast<T*>(a.dx) + (r0 + grp) * a.dx_stride;
    bool any = false;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (a.dx && in[k] && !live[k]) zero_row<T, VEC, NV, G, STREAM>(dx0 + k * RB * a.dx_stride, dim, lane);
      any |= live[k];
    }
    if (!__any(any)) return;  // padding; G > 64: the whole block agrees
    float xh[R][E], g[R][E], sums[2 * R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      sums[2 * k] = sums[2 * k + 1] = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        raw_widen<T, VEC>(rx[k][i], &xh[k][i * VEC]);
        raw_widen<T, VEC>(rg[k][i], &g[k][i * VEC]);
      }
#pragma unroll
      for (int i = 0; i < E; ++i) {  // past dim and in dead rows dy = 0, and nothing adds up
        xh[k][i] = (xh[k][i] - mean[k]) * rstd[k];
        dw[i] += g[k][i] * xh[k][i];
        db[i] += g[k][i];
        g[k][i] *= w[i];
        sums[2 * k] += g[k][i];
        sums[2 * k + 1] += g[k][i] * xh[k][i];
      }
    }
    if (a.dx) {
      row_sums<G, 2 * R>(sums, sh[turn]);
      turn ^= 1;  // a wave a turn ahead writes the other half
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (!live[k]) continue;
        const float mg = sums[2 * k] * inv_d, mgx = sums[2 * k + 1] * inv_d;
        T* dx = dx0 + k * RB * a.dx_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + lane) * VEC;
          if (c >= dim) continue;
          float o[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const int j = i * VEC + e;
            o[e] = rstd[k] * (g[k][j] - mg - xh[k][j] * mgx);
          }
          piece_store<T, VEC, STREAM>(dx + c, o);
        }
      }
    }
  };
  int64_t r0 = static_cast<int64_t>(blockIdx.x) * RB * R;
  Rows cur;
  if (kAhead) {
    load_bytes(r0);
    load_rows(r0, cur);
    load_bytes(r0 + step);
  }
  for (; r0 < a.rows; r0 += step) {
    if (kAhead) {
      Rows next;
      load_rows(r0 + step, next);
      load_bytes(r0 + 2 * step);
      work(r0, cur);
      cur = next;
    } else {
      load_bytes(r0);
      load_rows(r0, cur);
      work(r0, cur);
    }
  }
  if (!a.part) return;
  float* out = a.part + static_cast<int64_t>(blockIdx.x) * 2 * dim;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    float(&s)[E] = half ? db : dw;
    if (G < kBlock) {
#pragma unroll
      for (int i = 0; i < E; ++i) {  // the groups of the wave
        if (G <= 8) s[i] += __shfl_xor(s[i], 8, kWave);
        if (G <= 16) s[i] += __shfl_xor(s[i], 16, kWave);
        if (G <= 32) s[i] += __shfl_xor(s[i], 32, kWave);
      }
      const int l = threadIdx.x & (kWave - 1);
      __syncthreads();
      if (wave > 0 && l < GW)
#pragma unroll
        for (int i = 0; i < E; ++i) cols[wave - 1][i * GW + l] = s[i];
      __syncthreads();
      if (wave == 0 && l < GW)
#pragma unroll
        for (int i = 0; i < E; ++i)
#pragma unroll
          for (int k = 0; k < kWaves - 1; ++k) s[i] += cols[k][i * GW + l];
    }
    if (threadIdx.x < G)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int c = (i * G + lane) * VEC + e;
          if (c < dim) out[half * dim + c] = s[i * VEC + e];
        }
  }
}

template <typename T, int VEC, int NV, int G, int R>
void fwd_rows(const NormArgs& a, hipStream_t s) {
  // one pass per block, up to the 2^32 threads that a launch stays below; element-wise
  // parameter loads are shared by more rows
  const unsigned grid = grid_for(a.rows, kBlock / G * R, VEC > 1 ? 1 << 23 : 1 << 13);
  if (VEC > 1 && a.stream) k_ln_fwd<T, VEC, NV, G, R, (VEC > 1)><<<grid, kBlock, 0, s>>>(a);
  else k_ln_fwd<T, VEC, NV, G, R, false><<<grid, kBlock, 0, s>>>(a);
}
template <typename T, int VEC, int NV, int G, int R>
void bwd_rows(const NormArgs& a, hipStream_t s) {
  if (VEC > 1 && a.stream) k_ln_bwd<T, VEC, NV, G, R, (VEC > 1)><<<static_cast<unsigned>(a.nparts), kBlock, 0, s>>>(a);
  else k_ln_bwd<T, VEC, NV, G, R, false><<<static_cast<unsigned>(a.nparts), kBlock, 0, s>>>(a);
}

// Lanes per row: as few as hold it with one piece each, up to a wave; a wave
// then takes up to 16 elements per lane (8 without 16-byte pieces), a block
// the rows above that, up to 8192.
#define RS_NORM_ROWS(F)                                              \
  do {                                                               \
    const int64_t n = a.dim;                                         \
    if (wide) {                                                      \
      if constexpr (sizeof(T) == 2) {                                \
        if (n <= 64) F<T, 8, 1, 8, 2>(a, s);                         \
        else if (n <= 128) F<T, 8, 1, 16, 2>(a, s);                  \
        else if (n <= 256) F<T, 8, 1, 32, 2>(a, s);                  \
        else if (n <= 512) F<T, 8, 1, 64, 2>(a, s);                  \
        else if (n <= 1024) F<T, 8, 2, 64, 1>(a, s);                 \
        else if (n <= 2048) F<T, 8, 1, 256, 2>(a, s);                \
        else if (n <= 4096) F<T, 8, 2, 256, 1>(a, s);                \
        else F<T, 8, 4, 256, 1>(a, s);                               \
      } else {                                                       \
        if (n <= 32) F<T, 4, 1, 8, 2>(a, s);                         \
        else if (n <= 64) F<T, 4, 1, 16, 2>(a, s);                   \
        else if (n <= 128) F<T, 4, 1, 32, 2>(a, s);                  \
        else if (n <= 256) F<T, 4, 1, 64, 2>(a, s);                  \
        else if (n <= 512) F<T, 4, 2, 64, 2>(a, s);                  \
        else if (n <= 1024) F<T, 4, 4, 64, 1>(a, s);                 \
        else if (n <= 2048) F<T, 4, 2, 256, 2>(a, s);                \
        else if (n <= 4096) F<T, 4, 4, 256, 1>(a, s);                \
        else F<T, 4, 8, 256, 1>(a, s);                               \
      }                                                              \
    } else {                                                         \
      if (n <= 8) F<T, 1, 1, 8, 4>(a, s);                            \
      else if (n <= 32) F<T, 1, 1, 32, 4>(a, s);                     \
      else if (n <= 64) F<T, 1, 1, 64, 4>(a, s);                     \
      else if (n <= 128) F<T, 1, 2, 64, 2>(a, s);                    \
      else if (n <= 256) F<T, 1, 4, 64, 2>(a, s);                    \
      else if (n <= 512) F<T, 1, 8, 64, 1>(a, s);                    \
      else if (n <= 1024) F<T, 1, 4, 256, 2>(a, s);                  \
      else if (n <= 2048) F<T, 1, 8, 256, 1>(a, s);                  \
      else if (n <= 4096) F<T, 1, 16, 256, 1>(a, s);                 \
      else F<T, 1, 32, 256, 1>(a, s);                                \
    }                                                                \
  } while (0)

constexpr int64_t kRegDim = 8192;  // wider rows do not stay in registers

// Whether every row starts at a multiple of 16 bytes and is one long.
template <typename T>
bool rows16(const void* p, int64_t stride, int64_t dim) {
  constexpr int64_t kPer = 16 / sizeof(T);
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % kPer == 0 && dim % kPer == 0;
}

template <typename T>
hipError_t fwd(const NormArgs& a, hipStream_t s) {
  const bool wide = rows16<T>(a.x, a.x_stride, a.dim) && rows16<T>(a.y, a.y_stride, a.dim);
  if (a.dim > kRegDim) k_ln_fwd_any<T><<<grid_for(a.rows, 1, 1 << 16), kBlock, 0, s>>>(a);
  else RS_NORM_ROWS(fwd_rows);
  return hipGetLastError();
}

template <typename T>
hipError_t bwd(const NormArgs& a, hipStream_t s) {
  const bool wide = rows16<T>(a.x, a.x_stride, a.dim) && rows16<T>(a.dy, a.dy_stride, a.dim) &&
                    (!a.dx || rows16<T>(a.dx, a.dx_stride, a.dim));
  if (a.dim > kRegDim) {
    if (a.dx) k_ln_dx_any<T><<<grid_for(a.rows, 1, 1 << 16), kBlock, 0, s>>>(a);
    if (a.part) {
      const dim3 g(grid_for(a.dim, kBlock, 1ll << 31), static_cast<unsigned>(a.nparts));
      k_ln_cols_any<T><<<g, kBlock, 0, s>>>(a);
    }
  } else {
    RS_NORM_ROWS(bwd_rows);
  }
  if (a.part) 
    k_ln_cols_finish<<<grid_for(2 * a.dim, kFinishCols, 1ll << 31), kFinishCols * kFinishRows, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

int norm_parts(int64_t rows, int64_t dim) {
  const int64_t per = dim <= 256 ? 64 : dim <= 1024 ? 16 : 8;
  const int64_t most = dim <= 1024 ? 1024 : 512;
  const int64_t p = (rows + per - 1) / per;
  return static_cast<int>(p < 1 ? 1 : p > most ? most : p);
}

bool norm_param16(const void* weight, const void* bias) {
  return reinterpret_cast<uintptr_t>(weight) % 16 == 0 && reinterpret_cast<uintptr_t>(bias) % 16 == 0;
}

// Outputs larger than the L2 caches are stored past them: nothing of them
// would be left there for a reader, and the lines written back under the next
// kernel slow it.  Forward / backward of 65536 rows of 1024 bf16 (134 MB each)
// 51 / 81 us with plain stores, 42 / 67 us so.
bool norm_stream(int64_t rows, int64_t dim, bool bf16) { return rows * dim * (bf16 ? 2 : 4) > (int64_t(32) << 20); }

hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? fwd<uint16_t>(a, s) : fwd<float>(a, s);
}

hipError_t launch_norm_bwd(const NormArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? bwd<uint16_t>(a, s) : bwd<float>(a, s);
}

}  // namespace rs
