// Declarations shared by the sequence operators' kernels (layer norm and
// attention over ragged sequences) and their C ABI entry points.
#pragma once

#include "rs_internal.h"

namespace rs {

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------

// Strides are in elements; weight, bias and their gradients are bf16 where
// param_bf16 is set, else fp32.  Null pointers: weight 1, bias 0, no mask, no
// statistics wanted, a gradient not wanted.
struct NormArgs {
  int64_t rows, dim;
  float eps;
  bool param_bf16;
  bool stream;   // y / dx is stored past the caches
  bool param16;  // weight and bias start at multiples of 16 bytes
  const void* x;
  int64_t x_stride;
  const void *weight, *bias;
  const uint8_t* mask;
  // forward
  void* y;
  int64_t y_stride;
  float *mean_out, *rstd_out;
  // backward
  const void* dy;
  int64_t dy_stride;
  const float *mean, *rstd;
  void* dx;
  int64_t dx_stride;
  void *dweight, *dbias;
  float* part;  // [nparts][2 dim] partial column sums
  int nparts;
};

// Partial sums of dw and db: the rows of each are added by one block.
int norm_parts(int64_t rows, int64_t dim);
bool norm_stream(int64_t rows, int64_t dim, bool bf16);
bool norm_param16(const void* weight, const void* bias);
hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs& a, bool bf16, hipStream_t s);

// ---------------------------------------------------------------------------
// attention over ragged sequences
// ---------------------------------------------------------------------------

// Element strides of a [rows][heads][d] tensor whose d is contiguous.
struct HeadRows {
  const void* p;
  int64_t row, head;
};

struct AttnArgs {
  HeadRows q, k, v;
  // the launch's first block of all: HIP takes fewer than 2^32 threads along an axis
  uint32_t block0, blocks;
  const int64_t *q_off, *kv_off, *prefix;
  const float* slopes;
  int64_t q_rows, kv_rows, q_pad, kv_pad;
  int seqs, hq, hkv, group, d, causal;
  bool bf16;
  float scale, cap;
  // outputs (and the backward's inputs): contiguous [rows][heads][d]
  void* out;
  void* rest;  // what rounding to bf16 took from out, in bf16; null: not wanted
  float* lse;  // [q_rows][hq], natural logarithm
  // forward split along the keys (chunk > 0): chunks of that many keys, partial
  // results of up to part_rows rows of each block
  int chunk, row_tiles, part_rows;
  bool few;  // at most 32 narrow rows a sequence and key head
  float *part_o, *part_ml;
  // backward
  const void *o, *o_rest, *dout;
  const float* lse_in;
  void *dq, *dk, *dv;
  float *dslopes, *stat, *slope_part;
};

// Fills the split of the forward (chunk 0: none) for at most max_q queries a
// sequence (0: unknown); returns the workspace bytes its parts need, the
// probabilities' sums and maxima after the first *ml_at of them.
size_t plan_attn_split(AttnArgs* a, int64_t max_q, size_t* ml_at);
hipError_t launch_attn_fwd(const AttnArgs& a, bool bf16, hipStream_t s);
// Words per query row and head that the backward's first pass leaves for its second.
constexpr int kAttnStats = 4;
hipError_t launch_attn_bwd(const AttnArgs& a, bool bf16, hipStream_t s);
// Blocks of the pass over query rows (each leaves one partial sum per head
// of the slopes' gradient).
int64_t attn_row_tiles(const AttnArgs& a);

}  // namespace rs
