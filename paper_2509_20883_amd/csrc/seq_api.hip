// C ABI of the sequence operators (declared in include/recis_mi355x.h):
// argument checks, workspace layout and dispatch to the kernels.
#include <hip/hip_runtime.h>

#include <string>

#include "recis_mi355x.h"
#include "seq_internal.h"

using namespace rs;

namespace {

rs_status fail(rs_status st, const char* msg) { return set_last_error(st, msg); }

#define RS_HIP(call)                                                                   \
  do {                                                                                 \
    const hipError_t e_ = (call);                                                      \
    if (e_ != hipSuccess) return fail(RS_EHIP, hipGetErrorString(e_));                  \
  } while (0)

constexpr uintptr_t kAlign = 256;

bool valid_dtype(int32_t t) { return t == RS_F32 || t == RS_BF16; }

bool valid_norm(int64_t rows, int64_t dim) {
  return rows >= 0 && rows < (int64_t(1) << 31) && dim >= 1 && dim <= (int64_t(1) << 24);
}

bool valid_stride(int64_t stride, int64_t width) { return stride >= width && stride < (int64_t(1) << 32); }

}  // namespace

extern "C" {

rs_status layer_norm_fwd(const void* x, int64_t rows, int64_t dim, int64_t x_stride, int32_t dtype,
                         const void* weight, const void* bias, int32_t param_dtype, double eps, const uint8_t* mask,
                         void* y, int64_t y_stride, float* mean, float* rstd, rs_stream stream) {
  if (!valid_norm(rows, dim)) return fail(RS_EINVAL, "rows must be in [0, 2^31) and dim in [1, 2^24]");
  if (!valid_dtype(dtype) || !valid_dtype(param_dtype)) return fail(RS_EINVAL, "bad dtype or param_dtype");
  if (!valid_stride(x_stride, dim) || !valid_stride(y_stride, dim)) return fail(RS_EINVAL, "strides must be in [dim, 2^32)");
  if (!(eps >= 0.0)) return fail(RS_EINVAL, "eps must be >= 0");
  if (rows == 0) return RS_OK;
  if (!x || !y) return fail(RS_EINVAL, "null x or y");
  NormArgs a{};
  a.rows = rows;
  a.dim = dim;
  a.eps = static_cast<float>(eps);
  a.param_bf16 = param_dtype == RS_BF16;
  a.x = x;
  a.x_stride = x_stride;
  a.weight = weight;
  a.bias = bias;
  a.mask = mask;
  a.y = y;
  a.y_stride = y_stride;
  a.mean_out = mean;
  a.rstd_out = rstd;
  RS_HIP(launch_norm_fwd(a, dtype == RS_BF16, static_cast<hipStream_t>(stream)));
  return RS_OK;
}

size_t layer_norm_bwd_workspace_bytes(int64_t rows, int64_t dim) {
  if (!valid_norm(rows, dim)) return 0;
  return sizeof(float) * 2 * static_cast<size_t>(norm_parts(rows, dim)) * static_cast<size_t>(dim);
}

rs_status layer_norm_bwd(const void* dy, int64_t dy_stride, const void* x, int64_t rows, int64_t dim,
                         int64_t x_stride, int32_t dtype, const void* weight, int32_t param_dtype,
                         const uint8_t* mask, const float* mean, const float* rstd, void* dx, int64_t dx_stride,
                         void* dweight, void* dbias, void* workspace, size_t workspace_bytes, rs_stream stream) {
  if (!valid_norm(rows, dim)) return fail(RS_EINVAL, "rows must be in [0, 2^31) and dim in [1, 2^24]");
  if (!valid_dtype(dtype) || !valid_dtype(param_dtype)) return fail(RS_EINVAL, "bad dtype or param_dtype");
  if (!valid_stride(x_stride, dim) || !valid_stride(dy_stride, dim) || (dx && !valid_stride(dx_stride, dim)))
    return fail(RS_EINVAL, "strides must be in [dim, 2^32)");
  if (rows > 0 && (!dy || !x || !mean || !rstd)) return fail(RS_EINVAL, "null dy, x, mean or rstd");
  NormArgs a{};
  if (dweight || dbias) {
    if (!workspace || workspace_bytes < layer_norm_bwd_workspace_bytes(rows, dim))
      return fail(RS_EINVAL, "workspace missing or too small");
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return fail(RS_EINVAL, "workspace must be 256-byte aligned");
    a.part = static_cast<float*>(workspace);
    a.nparts = norm_parts(rows, dim);
  }
  a.rows = rows;
  a.dim = dim;
  a.param_bf16 = param_dtype == RS_BF16;
  a.x = x;
  a.x_stride = x_stride;
  a.weight = weight;
  a.mask = mask;
  a.dy = dy;
  a.dy_stride = dy_stride;
  a.mean = mean;
  a.rstd = rstd;
  a.dx = dx;
  a.dx_stride = dx_stride;
  a.dweight = dweight;
  a.dbias = dbias;
  RS_HIP(launch_norm_bwd(a, dtype == RS_BF16, static_cast<hipStream_t>(stream)));
  return RS_OK;
}

}  // extern "C"
