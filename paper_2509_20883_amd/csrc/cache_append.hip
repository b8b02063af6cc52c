// The paged sequence cache: new tokens in (with the rotation by their position)
// and rows out (gfx950).
//
// Rotation.  Columns (a, b) of a head turn by the angle p f: a' = a cos - b sin,
// b' = b cos + a sin.  f is held as a 64-bit fraction of a turn, so p f modulo a
// turn is one whole-number product, exact to 2^-33 turns at position 2^31 (an
// fp32 angle is off by 0.06 at 10^6).  Sine, cosine and the turn are taken in
// 64 bits and rounded once, to the model's type: a key that rounds the other way
// may fall across a border of the codes, and vector products of 64 bits issue as
// fast as those of 32.
//
// A full page is coded from the tokens in the model's type, those of its open
// page and the new ones, so the cache does not depend on how the tokens were
// cut into calls.  A page's tokens stay in LDS between the rotation, the
// maximum and the codes: inputs are read once and codes written once, in whole
// 1 KiB stores a wave.
#include <hip/hip_runtime.h>

#include "cache_common.h"

namespace rs {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Sine and cosine of a turn's fraction.  The quarter turns are taken off first;
// |x| <= pi / 4 then, and the series end at 8e-20.
__device__ inline void sincos_turn(uint64_t phase, double& s, double& c) {
  const uint64_t q = (phase + (uint64_t(1) << 61)) >> 62;  // nearest quarter
  const double x = static_cast<double>(static_cast<int64_t>(phase - (q << 62))) * (6.283185307179586477 * 0x1p-64);
  const double u = x * x;
  double a = 1.0 / 355687428096000.0;  // 1 / 17!
  a = fma(a, -u, 1.0 / 1307674368000.0);
  a = fma(a, -u, 1.0 / 6227020800.0);
  a = fma(a, -u, 1.0 / 39916800.0);
  a = fma(a, -u, 1.0 / 362880.0);
  a = fma(a, -u, 1.0 / 5040.0);
  a = fma(a, -u, 1.0 / 120.0);
  a = fma(a, -u, 1.0 / 6.0);
  a = fma(a, -u, 1.0) * x;
  double b = 1.0 / 20922789888000.0;  // 1 / 16!
  b = fma(b, -u, 1.0 / 87178291200.0);
  b = fma(b, -u, 1.0 / 479001600.0);
  b = fma(b, -u, 1.0 / 3628800.0);
  b = fma(b, -u, 1.0 / 40320.0);
  b = fma(b, -u, 1.0 / 720.0);
  b = fma(b, -u, 1.0 / 24.0);
  b = fma(b, -u, 0.5);
  b = fma(b, -u, 1.0);
  const double s1 = q & 1 ? b : a, c1 = q & 1 ? a : b;
  s = q & 2 ? -s1 : s1;
  c = (q + 1) & 2 ? -c1 : c1;
}

struct Angle {
  double s, c;
};
__device__ inline Angle angle_of(uint64_t phase) {
  Angle g;
  sincos_turn(phase, g.s, g.c);
  return g;
}
// A pair of columns turned, in the model's type.
__device__ inline void turn(const Angle& g, uint16_t& a, uint16_t& b) {
  const double x = bf16_to_f32(a), y = bf16_to_f32(b);
  a = f32_to_bf16(static_cast<float>(x * g.c - y * g.s));
  b = f32_to_bf16(static_cast<float>(y * g.c + x * g.s));
}
__device__ inline void turn(const Angle& g, float& a, float& b) {
  const double x = a, y = b;
  a = static_cast<float>(x * g.c - y * g.s);
  b = static_cast<float>(y * g.c + x * g.s);
}

__device__ inline float to_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ inline float to_f32(float x) { return x; }

// rne(x / s) exactly: the product by the reciprocal, then the remainder decides.
__device__ inline int code_i8(float x, float s, float inv) {
  float n = rintf(x * inv);
  const float e = fmaf(-n, s, x), half = 0.5f * s;
  if (fabsf(e) > half) n += copysignf(1.0f, e);
  else if (fabsf(e) == half && (static_cast<int>(n) & 1)) n += copysignf(1.0f, e);
  return static_cast<int>(fminf(fmaxf(n, -127.0f), 127.0f));
}

template <bool E4M3>
__device__ inline uint32_t codes4(const float (&x)[4], float s, float inv) {
  if (E4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true));
  }
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) w |= (static_cast<uint32_t>(code_i8(x[i], s, inv)) & 255u) << 8 * i;
  return w;
}

// Row stride of a page in LDS: 16 bytes past the columns, so that 16 tokens at
// one column chunk lie in different banks.
template <typename T>
__host__ __device__ inline int lds_stride(int d) {
  return d * static_cast<int>(sizeof(T)) + 16;
}

// The pairs of columns that turn: pair i is columns step i and step i + apart; a
// row's pairs take `lanes` lanes.
struct RotPairs {
  int count, lanes, step, apart;
  __device__ inline explicit RotPairs(const CacheAppend& a) {
    count = a.rotary / 2;
    lanes = count <= 1 ? 1 : 1 << (32 - __builtin_clz(count - 1));
    step = a.next ? 2 : 1;
    apart = a.next ? 1 : count;
  }
};

// Page number n of a sequence that holds tokens [held, end) after the call: coded
// if it is full, else its new tokens put into the open page.
template <typename T, bool E4M3, int NT>
__device__ __forceinline__ void append_page(const CacheAppend& a, char* lds, uint32_t* sh_top, float* sh_low, float* sh_high,
                                            int s, int kvh, int side, int slot, const SeqSpan& span, int64_t held,
                                            int64_t end, int64_t n) {
  constexpr int kPer = 16 / sizeof(T);
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int d = c.d, P = 1 << c.plog, W = d <= 32 ? 32 : d <= 64 ? 64 : 128;
  const RotPairs rp(a);
  const int half_rot = rp.count, pw = rp.lanes, ca = rp.step, cb = rp.apart;
  const int64_t first = n << c.plog;
  const bool full = first + P <= end;
  const int old = static_cast<int>(max(held - first, int64_t(0)));               // tokens the open page holds
  const int last = static_cast<int>(min(end - first, static_cast<int64_t>(P)));  // tokens the page holds now
  const int page = full ? cache_page(c, s, n) : -1;
  if ((full ? page < 0 : slot < 0) || (old > 0 && slot < 0)) return;  // block-uniform

  const int stride = lds_stride<T>(d), cpr = d / kPer;  // bytes, 16-byte chunks of a row
  const int cw = cpr <= 1 ? 1 : 1 << (32 - __builtin_clz(cpr - 1));
  const HeadRows& src = side ? a.v : a.k;
  const T* fresh = static_cast<const T*>(src.p) + (span.start + first - held) * src.row + kvh * src.head;  // of token 0
  T* open = slot < 0 ? nullptr : static_cast<T*>(c.open) + open_at(c, slot, n, kvh, side);
  const int t0 = full ? 0 : old;
  {
    const int ch = threadIdx.x & (cw - 1), per = NT / cw;
    if (ch < cpr)
      for (int t = t0 + threadIdx.x / cw; t < last; t += per) {
        const T* from = t < old ? open + t * d : fresh + t * src.row;
        *reinterpret_cast<u32x4*>(lds + t * stride + ch * 16) = *reinterpret_cast<const u32x4*>(from + ch * kPer);
      }
  }
  __syncthreads();
  if (side == 0 && half_rot > 0) {
    const int f = threadIdx.x & (pw - 1), per = NT / pw;
    if (f < half_rot) {
      const uint64_t step = a.turns[f];
      for (int t = max(t0, old) + threadIdx.x / pw; t < last; t += per) {
        const Angle g = angle_of(static_cast<uint64_t>(first + t) * step);
        T* x = reinterpret_cast<T*>(lds + t * stride) + ca * f;
        turn(g, x[0], x[cb]);
      }
    }
    __syncthreads();
  }
  if (!full) {
    const int ch = threadIdx.x & (cw - 1), per = NT / cw;
    if (ch < cpr)
      for (int t = t0 + threadIdx.x / cw; t < last; t += per)
        *reinterpret_cast<u32x4*>(open + t * d + ch * kPer) = *reinterpret_cast<const u32x4*>(lds + t * stride + ch * 16);
    return;
  }

  // the largest magnitude, as bits: infinities and NaN lie above every number
  uint32_t top = 0;
  {
    const int ch = threadIdx.x & (cw - 1), per = NT / cw;
    if (ch < cpr)
      for (int t = threadIdx.x / cw; t < P; t += per) {
        const T* x = reinterpret_cast<const T*>(lds + t * stride + ch * 16);
#pragma unroll
        for (int i = 0; i < kPer; ++i) top = max(top, __float_as_uint(to_f32(x[i])) & 0x7FFFFFFFu);
      }
  }
#pragma unroll
  for (int i = kWave / 2; i > 0; i >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), i, kWave)));
  if (lane == 0) sh_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT / kWave; ++i) top = max(top, sh_top[i]);
  const bool bad = top >= 0x7F800000u;  // the page then reads as NaN throughout
  const float most = __uint_as_float(top);
  float scale, inv;
  if (E4M3) {
    const int k = bad ? 0 : unit_exp(most, 1.75f, 8);
    scale = exp2_int(k);
    inv = exp2_int(-k);
  } else {
    scale = bad ? 1.0f : fmaxf(most / 127.0f, 0x1p-126f);
    inv = 1.0f / scale;
  }
  uint8_t* data = c.data + cache_at(c, page, kvh, side, W);
  if (side == 0) {
    for (int i = threadIdx.x; i < (W / 16) << c.plog; i += NT) {
      const int t = i & (P - 1), ch = i >> c.plog;
      u32x4 w = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!bad && ch * 16 + j * 4 < d) {
          const T* x = reinterpret_cast<const T*>(lds + t * stride) + ch * 16 + j * 4;
          const float y[4] = {to_f32(x[0]), to_f32(x[1]), to_f32(x[2]), to_f32(x[3])};
          w[j] = codes4<E4M3>(y, scale, inv);
        }
      *reinterpret_cast<u32x4*>(data + i * 16) = w;
    }
  } else {
    for (int i = threadIdx.x; i < W << (c.plog - 4); i += NT) {
      const int col = i & (W - 1), t = i / W * 16;
      u32x4 w = {0, 0, 0, 0};
      if (!bad && col < d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = to_f32(reinterpret_cast<const T*>(lds + (t + j * 4 + e) * stride)[col]);
          w[j] = codes4<E4M3>(y, scale, inv);
        }
      *reinterpret_cast<u32x4*>(data + i * 16) = w;
    }
  }
  const int64_t at = static_cast<int64_t>(page) * c.hkv + kvh;
  if (threadIdx.x == 0) c.scales[at * 2 + side] = bad ? __uint_as_float(0x7FC00000u) : scale;

  if (side == 0 && c.bounds) {
    // column maxima and minima in units of a power of two, rounded outward
    const int k = bad ? 0 : unit_exp(most, 1.984375f, 6);
    const float unit_inv = exp2_int(-k);
    const int col = threadIdx.x & (W - 1), share = threadIdx.x / W, shares = NT / W;
    float high = -INFINITY, low = INFINITY;
    if (col < d)
      for (int t = share; t < P; t += shares) {
        const float x = to_f32(reinterpret_cast<const T*>(lds + t * stride)[col]);
        high = fmaxf(high, x);
        low = fminf(low, x);
      }
    sh_high[threadIdx.x] = high;
    sh_low[threadIdx.x] = low;
    __syncthreads();
    if (share == 0) {
      for (int i = 1; i < shares; ++i) {
        high = fmaxf(high, sh_high[i * W + col]);
        low = fminf(low, sh_low[i * W + col]);
      }
      int8_t* to = c.bounds + at * 2 * W + col;
      const bool none = bad || col >= d;
      to[0] = none ? 0 : static_cast<int8_t>(ceilf(high * unit_inv));
      to[W] = none ? 0 : static_cast<int8_t>(floorf(low * unit_inv));
      if (col == 0) c.units[at] = bad ? __uint_as_float(0x7FC00000u) : exp2_int(k);
    }
  }
}

// The grid: blocks of (touched page, key head, side), then blocks of four query
// rows, then blocks of NT sequences for their new lengths.
template <typename T, bool E4M3, int NT>
__global__ __launch_bounds__(NT) void k_cache_append(const CacheAppend a) {
  extern __shared__ __align__(16) char lds[];
  __shared__ uint32_t sh_top[NT / kWave];
  __shared__ float sh_low[NT], sh_high[NT];
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int d = c.d, P = 1 << c.plog;
  int64_t b = a.block0 + blockIdx.x;

  if (b >= a.page_units * c.hkv * 2) {
    b -= a.page_units * c.hkv * 2;
    if (b < a.q_units) {
      // a wave per query row
      int64_t u = b * (NT / kWave) + wave, token;
      int s;
      if (c.pad > 0) {
        if (u >= c.rows) return;
        s = static_cast<int>(u / c.pad);
        token = u - s * c.pad;
      } else {
        if (u >= c.rows + c.seqs) return;
        s = find_seq(c.off, c.seqs, 1, 1, u, token);
      }
      const SeqSpan span = seq_span(c.off, s, c.pad, c.rows);
      if (token < 0 || token >= (c.pad > 0 ? c.pad : int64_t(span.len))) return;
      const int64_t row = span.start + token;
      T* out = static_cast<T*>(a.q_out) + row * a.hq * d;
      if (token >= span.len) {  // past the sequence's end
        for (int i = lane; i < a.hq * d; i += kWave) out[i] = T(0);
        return;
      }
      const T* q = static_cast<const T*>(a.q.p) + row * a.q.row;
      const uint64_t p = static_cast<uint64_t>(max(c.lens[s], int64_t(0)) + token);
      const RotPairs rp(a);
      const int half_rot = rp.count, pw = rp.lanes, ca = rp.step, cb = rp.apart;
      const int f = lane & (pw - 1), sub = lane / pw, step = kWave / pw;
      if (half_rot > 0 && f < half_rot) {
        const Angle g = angle_of(p * a.turns[f]);
        for (int h = sub; h < a.hq; h += step) {
          T x = q[h * a.q.head + ca * f], y = q[h * a.q.head + ca * f + cb];
          turn(g, x, y);
          out[h * d + ca * f] = x;
          out[h * d + ca * f + cb] = y;
        }
      }
      const int rest = d - a.rotary;
      for (int h = 0; h < a.hq && rest > 0; ++h)
        for (int i = a.rotary + lane; i < d; i += kWave) out[h * d + i] = q[h * a.q.head + i];
      return;
    }
    b -= a.q_units;
    const int64_t s = b * NT + threadIdx.x;
    if (s < c.seqs) {
      const SeqSpan span = seq_span(c.off, static_cast<int>(s), c.pad, c.rows);
      a.new_lens[s] = max(c.lens[s], int64_t(0)) + span.len;
    }
    return;
  }

  // a touched page of one key head, its keys or its values
  const int side = static_cast<int>(b & 1);
  b >>= 1;
  const int kvh = static_cast<int>(b % c.hkv);
  int64_t unit = b / c.hkv, tile;
  int s;
  if (c.pad > 0) {
    const int64_t per = (c.pad >> c.plog) + 2;
    s = static_cast<int>(unit / per);
    tile = unit - s * per;
  } else {
    s = find_pages(c.off, c.seqs, c.plog, unit, tile);
  }
  if (tile < 0) return;
  const SeqSpan span = seq_span(c.off, s, c.pad, c.rows);
  const int64_t held = max(c.lens[s], int64_t(0)), end = held + span.len;
  const int64_t n0 = held >> c.plog, n_end = end >> c.plog;
  if (span.len == 0 || (n0 + tile) << c.plog >= end) return;
  // The open page that the call ends in may lie where the one it starts in does.
  // The block that reads the first then writes the last, too, after it.
  const bool same = n_end > n0 && ((n_end - n0) & 1) == 0 && (held & (P - 1)) && (end & (P - 1));
  if (same && n0 + tile == n_end) return;
  const int slot = cache_slot(c, s);
  append_page<T, E4M3, NT>(a, lds, sh_top, sh_low, sh_high, s, kvh, side, slot, span, held, end, n0 + tile);
  if (same && tile == 0) {
    __syncthreads();
    append_page<T, E4M3, NT>(a, lds, sh_top, sh_low, sh_high, s, kvh, side, slot, span, held, end, n_end);
  }
}
__device__ inline void put(uint16_t* p, float x) { *p = f32_to_bf16(x); }
__device__ inline void put(float* p, float x) { *p = x; }

// Rows start[s] + i of sequence s as the cache holds them: a block per touched
// page and key head.
template <typename T, typename O, bool E4M3>
__global__ __launch_bounds__(kBlock) void k_cache_read(const CacheRead a, int64_t block0) {
  const CacheArgs& c = a.c;
  const int d = c.d, P = 1 << c.plog, W = d <= 32 ? 32 : d <= 64 ? 64 : 128;
  const int64_t b = block0 + blockIdx.x;
  const int kvh = static_cast<int>(b % c.hkv);
  int64_t tile;
  const int s = find_pages(c.off, c.seqs, c.plog, b / c.hkv, tile);
  if (tile < 0) return;
  const SeqSpan span = seq_span(c.off, s, 0, c.rows);
  const int64_t begin = a.start ? max(a.start[s], int64_t(0)) : 0, end = begin + span.len;
  const int64_t n = (begin >> c.plog) + tile, first = n << c.plog;
  if (first >= end) return;
  const int t0 = static_cast<int>(max(begin - first, int64_t(0))), t1 = static_cast<int>(min(end - first, static_cast<int64_t>(P)));
  const int len = cache_len(c, s);
  const bool full = first + P <= len;
  const int slot = cache_slot(c, s), page = full ? cache_page(c, s, n) : -1;
  const int64_t row0 = span.start + first - begin;  // of the page's token 0
  auto at = [&](void* base, int t) { return static_cast<O*>(base) + ((row0 + t) * c.hkv + kvh) * d; };
  if (!full || page < 0) {
    const int held = !full && slot >= 0 ? static_cast<int>(min(max(len - first, int64_t(0)), static_cast<int64_t>(t1))) : 0;
    for (int side = 0; side < 2; ++side) {
      const T* open = static_cast<const T*>(c.open) + (held > 0 ? open_at(c, slot, n, kvh, side) : 0);
      const int cols = d;
      for (int i = threadIdx.x; i < (t1 - t0) * cols; i += kBlock) {
        const int t = t0 + i / cols, col = i % cols;
        put(at(side ? a.v : a.k, t) + col, t < held ? to_f32(open[t * d + col]) : 0.0f);
      }
    }
    return;
  }
  const float* sc = c.scales + (static_cast<int64_t>(page) * c.hkv + kvh) * 2;
  const uint8_t* keys = c.data + cache_at(c, page, kvh, 0, W);
  for (int i = threadIdx.x; i < (W / 16) << c.plog; i += kBlock) {
    const int t = i & (P - 1), ch = i >> c.plog;
    if (t < t0 || t >= t1) continue;
    const u32x4 w = *reinterpret_cast<const u32x4*>(keys + i * 16);
    O* to = at(a.k, t) + ch * 16;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (ch * 16 + j * 4 < d)
#pragma unroll
        for (int e = 0; e < 4; ++e) put(to + j * 4 + e, code_value<E4M3>(static_cast<uint8_t>(w[j] >> 8 * e)) * sc[0]);
  }
  const uint8_t* values = c.data + cache_at(c, page, kvh, 1, W);
  for (int i = threadIdx.x; i < W << (c.plog - 4); i += kBlock) {
    const int col = i & (W - 1), t = i / W * 16;
    if (col >= d) continue;
    const u32x4 w = *reinterpret_cast<const u32x4*>(values + i * 16);
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (t + j >= t0 && t + j < t1)
        put(at(a.v, t + j) + col, code_value<E4M3>(static_cast<uint8_t>(w[j >> 2] >> 8 * (j & 3))) * sc[1]);
  }
}

constexpr int64_t kMostBlocks = int64_t(1) << 21;  // of a launch: fewer than 2^32 threads along an axis

template <typename T, bool E4M3, int NT>
hipError_t append(CacheAppend a, int bytes, hipStream_t s) {
  const bool rows = a.k.p != nullptr && a.c.rows > 0;
  const int64_t u = a.c.pad > 0 ? a.c.seqs * ((a.c.pad >> a.c.plog) + 2) : (a.c.rows >> a.c.plog) + 2 * int64_t(a.c.seqs);
  a.page_units = rows ? u : 0;
  a.q_units = a.q.p ? ((a.c.pad > 0 ? a.c.rows : a.c.rows + a.c.seqs) + NT / kWave - 1) / (NT / kWave) : 0;
  const int64_t lens = a.new_lens ? (a.c.seqs + NT - 1) / NT : 0;
  const int64_t blocks = a.page_units * a.c.hkv * 2 + a.q_units + lens;
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_cache_append<T, E4M3, NT>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {
    a.block0 = b;
    const int64_t now = blocks - b < kMostBlocks ? blocks - b : kMostBlocks;
    k_cache_append<T, E4M3, NT><<<static_cast<unsigned>(now), NT, bytes, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, bool E4M3>
hipError_t append_type(const CacheAppend& a, hipStream_t s) {
  const int bytes = lds_stride<T>(a.c.d) << a.c.plog;
  // a large page fills a CU's LDS by itself: more waves on it then
  return bytes > 65536 ? append<T, E4M3, 1024>(a, bytes, s) : append<T, E4M3, 256>(a, bytes, s);
}

template <typename T, typename O, bool E4M3>
hipError_t read_type(const CacheRead& a, hipStream_t s) {
  const int64_t blocks = ((a.c.rows >> a.c.plog) + 2 * int64_t(a.c.seqs)) * a.c.hkv;
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {
    const int64_t now = blocks - b < kMostBlocks ? blocks - b : kMostBlocks;
    k_cache_read<T, O, E4M3><<<static_cast<unsigned>(now), kBlock, 0, s>>>(a, b);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheAppend& a, bool bf16, bool e4m3, hipStream_t s) {
  if (bf16) return e4m3 ? append_type<uint16_t, true>(a, s) : append_type<uint16_t, false>(a, s);
  return e4m3 ? append_type<float, true>(a, s) : append_type<float, false>(a, s);
}

hipError_t launch_cache_read(const CacheRead& a, bool bf16, bool e4m3, hipStream_t s) {
  if (bf16) {
    if (a.out_bf16) return e4m3 ? read_type<uint16_t, uint16_t, true>(a, s) : read_type<uint16_t, uint16_t, false>(a, s);
    return e4m3 ? read_type<uint16_t, float, true>(a, s) : read_type<uint16_t, float, false>(a, s);
  }
  if (a.out_bf16) return e4m3 ? read_type<float, uint16_t, true>(a, s) : read_type<float, uint16_t, false>(a, s);
  return e4m3 ? read_type<float, float, true>(a, s) : read_type<float, float, false>(a, s);
}

}  // namespace rs
