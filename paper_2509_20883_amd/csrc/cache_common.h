// Device helpers of the paged sequence cache (gfx950): where things lie, and
// 8-bit codes as operands of the matrix instructions.
#pragma once

#include "attn_common.h"
#include "cache_internal.h"

namespace rs {

// Tokens that sequence s holds: lens[s], cut to what its table can name.
__device__ inline int cache_len(const CacheArgs& c, int s) {
  return static_cast<int>(min(max(c.lens[s], int64_t(0)), min(c.width << c.plog, int64_t(0x7FFFFF00))));
}
// The slot of its open pages, or -1.
__device__ inline int cache_slot(const CacheArgs& c, int s) {
  const int64_t x = c.slot_of ? static_cast<int64_t>(c.slot_of[s]) : s;
  return x >= 0 && x < c.slots ? static_cast<int>(x) : -1;
}
// The page that holds page number n of sequence s, or -1.
__device__ inline int cache_page(const CacheArgs& c, int s, int64_t n) {
  if (n < 0 || n >= c.width) return -1;
  const int32_t p = c.table[s * c.width + n];
  return p >= 0 && p < c.pages ? p : -1;
}
// First byte of a page's keys (side 0) or values (side 1).
__device__ inline int64_t cache_at(const CacheArgs& c, int page, int kvh, int side, int W) {
  return ((static_cast<int64_t>(page) * c.hkv + kvh) * 2 + side) * (static_cast<int64_t>(W) << c.plog);
}
// First element of the open page of page number n.
__device__ inline int64_t open_at(const CacheArgs& c, int slot, int64_t n, int kvh, int side) {
  return ((((static_cast<int64_t>(slot) * 2 + (n & 1)) * c.hkv + kvh) * 2 + side) << c.plog) * c.d;
}

// Block numbers over the pages that a sequence's rows touch: off[s] / P + 2 s on,
// enough for rows that start anywhere in a page (n rows touch at most n / P + 2).
__device__ inline int find_pages(const int64_t* __restrict__ off, int seqs, int plog, int64_t b, int64_t& tile) {
  const int lane = threadIdx.x & (kWave - 1);
  int lo = 0, n = seqs;
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave;
    const int s = lane * step;
    const bool below = s < n && (max(off[lo + s], int64_t(0)) >> plog) + 2 * int64_t(lo + s) <= b;
    const int c = max(1, static_cast<int>(__popcll(__ballot(below))));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  tile = b - ((max(off[lo], int64_t(0)) >> plog) + 2 * int64_t(lo));
  return lo;
}

// The sequence of block b and its tile there, for tiles of 1 << log rows: sequence s from
// off[s] >> log on, and s more as each may end within a tile; single rows never do, so
// there `rows` blocks are enough.
__device__ inline int find_tile(const int64_t* __restrict__ off, int seqs, int group, int log, uint32_t b, int64_t& tile) {
  const int lane = threadIdx.x & (kWave - 1);
  int lo = 0, n = seqs;
  while (n > 1) {
    const int step = static_cast<int>(static_cast<uint32_t>(n + kWave - 1) / kWave);
    const int s = lane * step;
    const bool below = s < n && (max(off[lo + s], int64_t(0)) * group >> log) + (log ? lo + s : 0) <= static_cast<int64_t>(b);
    const int c = max(1, static_cast<int>(__popcll(__ballot(below))));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  tile = static_cast<int64_t>(b) - ((max(off[lo], int64_t(0)) * group >> log) + (log ? lo : 0));
  return lo;
}

// The exponent k, from -126 on, of the least power of two with top <= most 2^k,
// for most = mant 2^exp2 (1 <= mant < 2).
__device__ inline int unit_exp(float top, float mant, int exp2) {
  const uint32_t b = __float_as_uint(top);
  const float m = __uint_as_float((b & 0x007FFFFFu) | 0x3F800000u);
  const int e = static_cast<int>(b >> 23) - 127;
  return max(-126, m <= mant ? e - exp2 : e - exp2 + 1);
}
__device__ inline float exp2_int(int k) { return __uint_as_float(static_cast<uint32_t>(k + 127) << 23); }

// Two signed bytes of a word as bf16. Written out, since the compiler else turns
// all the bytes of a step into floats first and spills them.
template <int HIGH>
__device__ inline uint32_t pack_i8(uint32_t x) {
  float a = 0.0f, b = 0.0f;
#if defined(__HIP_DEVICE_COMPILE__)
  if (HIGH) {
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(a) : "v"(x));
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(b) : "v"(x));
  } else {
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(a) : "v"(x));
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(b) : "v"(x));
  }
#endif
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);  // whole numbers: no rounding
}

// Eight codes as bf16, where both kinds are exact; e4m3 times a power of two, which
// the conversion takes along.
template <bool E4M3>
__device__ inline bf16x8 codes8(uint32_t lo, uint32_t hi, float scale) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 w;
  if (E4M3) {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  } else {
    w[0] = pack_i8<0>(lo);
    w[1] = pack_i8<1>(lo);
    w[2] = pack_i8<0>(hi);
    w[3] = pack_i8<1>(hi);
  }
  return __builtin_bit_cast(bf16x8, w);
}

// One code's value.
template <bool E4M3>
__device__ inline float code_value(uint8_t c) {
  if (!E4M3) return static_cast<float>(static_cast<int8_t>(c));
  return __builtin_amdgcn_cvt_f32_fp8(c, 0);
}

}  // namespace rs
