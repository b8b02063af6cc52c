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

// Any width: a block per row that passes over it three times (mean, variance,
// result); after the first the row comes from the caches.
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

// Adds up the partial sums: 16 columns per block, 16 threads per column, in a
// fixed order, so the result does not change from run to run.
__global__ __launch_bounds__(kBlock) void k_ln_cols_finish(const NormArgs a) {
  constexpr int C = 16, R = kBlock / C;
  __shared__ float sh[R][C + 1];
  const int64_t c = static_cast<int64_t>(blockIdx.x) * C + threadIdx.x % C;
  const int r = threadIdx.x / C;
  float s = 0.0f;
  if (c < 2 * a.dim)
    for (int p = r; p < a.nparts; p += R) s += a.part[static_cast<int64_t>(p) * 2 * a.dim + c];
  sh[r][threadIdx.x % C] = s;
  __syncthreads();
  if (r == 0 && c < 2 * a.dim) {
    float t = 0.0f;
#pragma unroll
    for (int k = 0; k < R; ++k) t += sh[k][threadIdx.x];
    void* out = c < a.dim ? a.dweight : a.dbias;
    const int64_t i = c < a.dim ? c : c - a.dim;
    if (out) {
      if (a.param_bf16) static_cast<uint16_t*>(out)[i] = f32_to_bf16(t);
      else static_cast<float*>(out)[i] = t;
    }
  }
}

template <typename T>
hipError_t fwd(const NormArgs& a, hipStream_t s) {
  k_ln_fwd_any<T><<<grid_for(a.rows, 1, 1 << 16), kBlock, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t bwd(const NormArgs& a, hipStream_t s) {
  if (a.dx) k_ln_dx_any<T><<<grid_for(a.rows, 1, 1 << 16), kBlock, 0, s>>>(a);
  if (a.dweight || a.dbias) {
    const dim3 g(grid_for(a.dim, kBlock, 1ll << 31), static_cast<unsigned>(a.nparts));
    k_ln_cols_any<T><<<g, kBlock, 0, s>>>(a);
    k_ln_cols_finish<<<grid_for(2 * a.dim, 16, 1ll << 31), kBlock, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

int norm_parts(int64_t rows, int64_t dim) {
  const int64_t p = (rows + 63) / 64;
  return static_cast<int>(p < 1 ? 1 : p > 1024 ? 1024 : p);
}

hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? fwd<uint16_t>(a, s) : fwd<float>(a, s);
}

hipError_t launch_norm_bwd(const NormArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? bwd<uint16_t>(a, s) : bwd<float>(a, s);
}

}  // namespace rs
