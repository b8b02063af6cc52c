// C ABI of the sequence operators (declared in include/recis_mi355x.h):
// argument checks, workspace layout and dispatch to the kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>
#include <vector>

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

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// An upper bound of the blocks of any launch.
int64_t attn_blocks(const rs_attn_desc& d) {
  const int64_t group = d.heads_q / d.heads_kv;
  const int64_t q = d.q_pad > 0 ? d.seqs * (d.q_pad * group / 128 + 1) : d.q_rows * group / 128 + d.seqs;
  const int64_t k = d.kv_pad > 0 ? d.seqs * (d.kv_pad / 64 + 1) : d.kv_rows / 64 + d.seqs;
  return std::max(q, k) * d.heads_kv;
}

// What is wrong with a descriptor, or null.
const char* check_attn(const rs_attn_desc* d) {
  if (!d) return "null descriptor";
  if (!valid_dtype(d->dtype)) return "bad dtype";
  if (d->heads_kv < 1 || d->heads_kv > 1024) return "heads_kv must be in [1, 1024]";
  if (d->heads_q < d->heads_kv || d->heads_q > 8192 || d->heads_q % d->heads_kv != 0)
    return "heads_q must be a multiple of heads_kv, at most 8192";
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8 != 0) return "head_dim must be a multiple of 8 in [8, 128]";
  if (d->reserved != 0) return "reserved must be 0";
  constexpr int64_t kMost = (int64_t(1) << 31) - 1024;  // a tile past the last row still counts in 32 bits
  if (d->seqs < 0 || d->seqs >= (int64_t(1) << 24)) return "seqs must be in [0, 2^24)";
  if (d->q_rows < 0 || d->q_rows >= kMost || d->q_rows * d->heads_q >= kMost) return "q_rows * heads_q must be below 2^31 - 1024";
  if (d->kv_rows < 0 || d->kv_rows >= kMost) return "kv_rows must be in [0, 2^31 - 1024)";
  if (d->q_pad < 0 || d->q_pad >= kMost || d->kv_pad < 0 || d->kv_pad >= kMost) return "pad lengths must be in [0, 2^31 - 1024)";
  if (d->q_pad > 0 && d->seqs * d->q_pad != d->q_rows) return "padded: q_rows must be seqs * q_pad";
  if (d->kv_pad > 0 && d->seqs * d->kv_pad != d->kv_rows) return "padded: kv_rows must be seqs * kv_pad";
  if (d->max_q < 0) return "max_q must be >= 0";
  const int64_t unit = d->dtype == RS_BF16 ? 8 : 4;
  for (const int64_t st : {d->q_stride, d->q_head_stride, d->k_stride, d->k_head_stride, d->v_stride, d->v_head_stride})
    if (st < 0 || st >= (int64_t(1) << 23) || st % unit != 0)
      return "strides must be multiples of 16 bytes in [0, 2^23) elements";
  // a wave's share of a step of packed rows, at most 16 tokens and a group of heads, is addressed with 31 bits
  const int64_t es = d->dtype == RS_BF16 ? 2 : 4;
  if ((64 * d->q_stride + d->heads_q / d->heads_kv * d->q_head_stride) * es >= kMost)
    return "64 rows and a group of heads of q must span less than 2^31 bytes";
  if (attn_blocks(*d) >= kMost) return "too many sequences, rows and key heads: below 2^31 blocks";
  // the kernels hold both, and their quotient, in fp32
  const float scale = static_cast<float>(d->scale), cap = static_cast<float>(d->softcap);
  if (!(d->scale > 0.0) || !(d->scale < 0x1p127)) return "scale must be > 0 and below 2^127";
  if (!(d->softcap >= 0.0) || !std::isfinite(d->softcap)) return "softcap must be finite and >= 0";
  if (d->softcap > 0.0 && (cap < FLT_MIN || !std::isfinite(scale / cap)))
    return "softcap and scale / softcap must be within fp32's range";
  return nullptr;
}

AttnArgs attn_args(const rs_attn_desc& d) {
  AttnArgs a{};
  a.q = HeadRows{nullptr, d.q_stride, d.q_head_stride};
  a.k = HeadRows{nullptr, d.k_stride, d.k_head_stride};
  a.v = HeadRows{nullptr, d.v_stride, d.v_head_stride};
  a.q_rows = d.q_rows;
  a.kv_rows = d.kv_rows;
  a.q_pad = d.q_pad;
  a.kv_pad = d.kv_pad;
  a.seqs = static_cast<int>(d.seqs);
  a.hq = d.heads_q;
  a.hkv = d.heads_kv;
  a.group = d.heads_q / d.heads_kv;
  a.d = d.head_dim;
  a.bf16 = d.dtype == RS_BF16;
  a.causal = d.causal != 0;
  a.scale = static_cast<float>(d.scale);
  // A score below 2^-13 of the cap is cap(x) to within fp32's rounding: past 2^100
  // every score is, and the cap's own products would leave fp32's range.
  a.cap = d.softcap < 0x1p100 ? static_cast<float>(d.softcap) : 0.0f;
  return a;
}

// Host check of the offsets: copies them back, so it synchronizes.
rs_status check_offsets(const rs_attn_desc& d, const int64_t* q_off, const int64_t* kv_off, hipStream_t s) {
  try {
    RS_HIP(hipStreamSynchronize(s));
    std::vector<int64_t> off(static_cast<size_t>(d.seqs) + 1);
    for (int side = 0; side < 2; ++side) {
      RS_HIP(hipMemcpy(off.data(), side ? kv_off : q_off, sizeof(int64_t) * off.size(), hipMemcpyDeviceToHost));
      if (off[0] != 0) return fail(RS_EINVAL, "offsets must start at 0");
      for (int64_t i = 0; i < d.seqs; ++i) {
        if (off[i + 1] < off[i]) return fail(RS_EINVAL, "offsets must be nondecreasing");
        if (side == 0 && d.max_q > 0 && off[i + 1] - off[i] > d.max_q && (d.q_pad == 0 || d.q_pad > d.max_q))
          return fail(RS_EINVAL, "a sequence has more than max_q queries");
      }
      if ((side ? d.kv_pad : d.q_pad) == 0 && off[d.seqs] != (side ? d.kv_rows : d.q_rows))
        return fail(RS_EINVAL, "packed offsets must end at the number of rows");
    }
  } catch (const std::bad_alloc&) {
    return fail(RS_ENOMEM, "no host memory for the offsets' check");
  }
  return RS_OK;
}

struct BwdWork {
  size_t slope_part, total;  // the rows' statistics come first
};
BwdWork bwd_work(const AttnArgs& a) {
  BwdWork w{};
  w.slope_part = align_up(kAttnStats * sizeof(float) * static_cast<size_t>(a.q_rows) * static_cast<size_t>(a.hq));
  w.total = w.slope_part + align_up(sizeof(float) * static_cast<size_t>(attn_row_tiles(a)) * static_cast<size_t>(a.hq));
  return w;
}

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
  a.stream = norm_stream(rows, dim, dtype == RS_BF16);
  a.x = x;
  a.x_stride = x_stride;
  a.weight = weight;
  a.bias = bias;
  a.param16 = norm_param16(weight, bias);
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
  }
  a.nparts = norm_parts(rows, dim);
  a.rows = rows;
  a.dim = dim;
  a.param_bf16 = param_dtype == RS_BF16;
  a.stream = norm_stream(rows, dim, dtype == RS_BF16);
  a.x = x;
  a.x_stride = x_stride;
  a.weight = weight;
  a.param16 = norm_param16(weight, nullptr);
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

size_t seq_attention_workspace_bytes(const rs_attn_desc* d, int32_t backward) {
  if (check_attn(d)) return 0;
  AttnArgs a = attn_args(*d);
  size_t at = 0;
  return backward ? bwd_work(a).total : plan_attn_split(&a, d->max_q, &at);
}

rs_status seq_attention_fwd(const rs_attn_desc* d, const void* q, const void* k, const void* v,
                            const int64_t* q_offsets, const int64_t* kv_offsets, const int64_t* prefix,
                            const float* slopes, void* out, void* rest, float* lse, void* workspace, size_t workspace_bytes,
                            int32_t validate, rs_stream stream) {
  if (const char* bad = check_attn(d)) return fail(RS_EINVAL, bad);
  if (!q_offsets || !kv_offsets) return fail(RS_EINVAL, "null offsets");
  if (d->q_rows > 0 && (!q || !out)) return fail(RS_EINVAL, "null q or out");
  if (d->kv_rows > 0 && (!k || !v)) return fail(RS_EINVAL, "null k or v");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(rest))
    return fail(RS_EINVAL, "q, k, v, out and rest must be 16-byte aligned");
  AttnArgs a = attn_args(*d);
  size_t ml_at = 0;
  const size_t need = plan_attn_split(&a, d->max_q, &ml_at);
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return fail(RS_EINVAL, "workspace missing or too small");
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return fail(RS_EINVAL, "workspace must be 256-byte aligned");
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + ml_at);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (validate) {
    const rs_status st = check_offsets(*d, q_offsets, kv_offsets, s);
    if (st != RS_OK) return st;
  }
  if (d->seqs == 0 || d->q_rows == 0) return RS_OK;
  a.q.p = q;
  a.k.p = k;
  a.v.p = v;
  a.q_off = q_offsets;
  a.kv_off = kv_offsets;
  a.prefix = d->causal ? prefix : nullptr;
  a.slopes = slopes;
  a.out = out;
  a.rest = d->dtype == RS_BF16 ? rest : nullptr;
  a.lse = lse;
  RS_HIP(launch_attn_fwd(a, d->dtype == RS_BF16, s));
  return RS_OK;
}

rs_status seq_attention_bwd(const rs_attn_desc* d, const void* q, const void* k, const void* v, const void* out,
                            const void* rest, const float* lse, const void* grad_out, const int64_t* q_offsets,
                            const int64_t* kv_offsets, const int64_t* prefix, const float* slopes, void* dq,
                            void* dk, void* dv, float* dslopes, void* workspace, size_t workspace_bytes,
                            int32_t validate, rs_stream stream) {
  if (const char* bad = check_attn(d)) return fail(RS_EINVAL, bad);
  if (!q_offsets || !kv_offsets) return fail(RS_EINVAL, "null offsets");
  if (d->q_rows > 0 && (!q || !out || !lse || !grad_out || !dq)) return fail(RS_EINVAL, "null q, out, lse, grad_out or dq");
  if (d->kv_rows > 0 && (!k || !v || !dk || !dv)) return fail(RS_EINVAL, "null k, v, dk or dv");
  if (dslopes && !slopes) return fail(RS_EINVAL, "dslopes needs slopes");
  for (const void* p : {q, k, v, out, rest, grad_out, static_cast<const void*>(dq), static_cast<const void*>(dk),
                        static_cast<const void*>(dv)})
    if (!aligned16(p)) return fail(RS_EINVAL, "q, k, v, out, rest, grad_out, dq, dk and dv must be 16-byte aligned");
  AttnArgs a = attn_args(*d);
  const BwdWork w = bwd_work(a);
  if (w.total > 0 && (!workspace || workspace_bytes < w.total)) return fail(RS_EINVAL, "workspace missing or too small");
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return fail(RS_EINVAL, "workspace must be 256-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (validate) {
    const rs_status st = check_offsets(*d, q_offsets, kv_offsets, s);
    if (st != RS_OK) return st;
  }
  a.q.p = q;
  a.k.p = k;
  a.v.p = v;
  a.q_off = q_offsets;
  a.kv_off = kv_offsets;
  a.prefix = d->causal ? prefix : nullptr;
  a.slopes = slopes;
  a.o = out;
  a.o_rest = d->dtype == RS_BF16 ? rest : nullptr;
  a.dout = grad_out;
  a.lse_in = lse;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dslopes = dslopes;
  uint8_t* base = static_cast<uint8_t*>(workspace);
  a.stat = reinterpret_cast<float*>(base);
  a.slope_part = dslopes ? reinterpret_cast<float*>(base + w.slope_part) : nullptr;
  RS_HIP(launch_attn_bwd(a, d->dtype == RS_BF16, s));
  return RS_OK;
}

}  // extern "C"
