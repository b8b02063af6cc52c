// The paged sequence cache: new tokens in (with the rotation by their position)
// and rows out (gfx950).
//
// Rotation.  Columns (a, b) of a head turn by the angle p f: a' = a cos - b sin,
// b' = b cos + a sin.  f is held as a 64-bit fraction of a turn, so p f modulo a
// turn is one whole-number product, exact to 2^-33 turns at position 2^31 (an
// fp32 angle is off by 0.06 at 10^6).  Sine, cosine and the turn are taken in
// 64 bits: a key that rounds the other way may fall across a border of the codes,
// and vector products of 64 bits issue as fast as those of 32.  The result is
// rounded to the model's type, to bf16 by way of fp32, as a conversion from 64 bits
// does it elsewhere: one value in 2^17 or so, within 2^-25 of itself of the middle
// between two bf16 numbers, goes to the other one.
//
// A full page is coded from the tokens in the model's type, those of its open
// page and the new ones, so the cache does not depend on how the tokens were
// cut into calls.  A page's tokens stay in LDS between the rotation, the
// maximum and the codes: inputs are read once and codes written once, in whole
// 1 KiB stores a wave.
//
// 24 histories of 17 to 8191 tokens (93 thousand rows of 8 query and 2 key heads of
// 128, bf16 to e4m3 with bounds, 524 MB moved): 133 us, 3.9 TB/s, where a plain copy
// of the queries' 380 MB takes 72. Query rows alone take 72 us, pages alone 54 to 64:
// a page waits for one thing after another (its sequence, its place, its tokens, then
// four steps with barriers between), and keys turn at 14 us of those. Blocks of
// both kinds mixed in the grid, the next row loaded a step ahead, angles without
// LDS bank conflicts: no change (126 to 128 where 125 was). One token of 256 users: 9.9 us, bound by
// latency. Reading the 24 histories back (143 MB moved): 25 us, 5.7 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_common.h"

namespace rs {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Sine and cosine of a turn's fraction.  The quarter turns are taken off first;
// |x| <= pi / 4 then; the first terms left out are 8e-20 (sine) and 2e-18 (cosine).
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
// The angle further on by another: off by 2^-53, where a series takes 15 times as
// many instructions.
__device__ inline void advance(Angle& g, const Angle& by) {
  const double s = fma(g.s, by.c, g.c * by.s);
  g.c = fma(g.c, by.c, -(g.s * by.s));
  g.s = s;
}
// The angles of one frequency at one position after another. A series every 16 positions,
// from there by fours, from a multiple of four by ones: an angle is a function of its
// position to the last bit, not of where a call, a tile or a thread began. (Which product
// is fused is written out, above and below: left to the compiler it is another one in
// another place.)
struct Turning {
  uint64_t turns;
  int64_t pos;
  Angle one, four, group, g;
  __device__ inline explicit Turning(uint64_t t) : turns(t) {
    one = four = angle_of(t);
    advance(four, one);
    const Angle two = four;
    advance(four, two);
  }
  __device__ inline void start(int64_t p) {
    pos = p;
    group = angle_of(static_cast<uint64_t>(p & ~int64_t(15)) * turns);
    for (int i = static_cast<int>(p >> 2 & 3); i > 0; --i) advance(group, four);
    g = group;
    for (int i = static_cast<int>(p & 3); i > 0; --i) advance(g, one);
  }
  // to the next position, not a multiple of 16
  __device__ inline void next() {
    ++pos;
    if (pos & 3) {
      advance(g, one);
    } else {
      advance(group, four);
      g = group;
    }
  }
};
// A pair of columns turned, in the model's type.
__device__ inline void turn(const Angle& g, uint16_t& a, uint16_t& b) {
  const double x = bf16_to_f32(a), y = bf16_to_f32(b);
  const uint32_t w = pack_bf16(static_cast<float>(fma(x, g.c, -(y * g.s))), static_cast<float>(fma(y, g.c, x * g.s)));
  a = static_cast<uint16_t>(w);
  b = static_cast<uint16_t>(w >> 16);
}
__device__ inline void turn(const Angle& g, float& a, float& b) {
  const double x = a, y = b;
  a = static_cast<float>(fma(x, g.c, -(y * g.s)));
  b = static_cast<float>(fma(y, g.c, x * g.s));
}

__device__ inline float to_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ inline float to_f32(float x) { return x; }

// rne(x / s) exactly: the product by the reciprocal, then the remainder decides (twice
// it against s: half of the least scales is not a number).
__device__ inline int code_i8(float x, float s, float inv) {
  float n = rintf(x * inv);
  const float e = 2.0f * fmaf(-n, s, x);
  if (fabsf(e) > s) n += copysignf(1.0f, e);
  else if (fabsf(e) == s && (static_cast<int>(n) & 1)) n += copysignf(1.0f, e);
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

// A page that fills while its first tokens are gone (they came for a slot outside the
// cache): what it held before, another sequence's maybe, goes, and a scale of 0, which
// no page of tokens has, says that there is nothing to see.
__device__ inline void lost_page(const CacheArgs& c, int page, int kvh, int side, int W) {
  const int64_t at = static_cast<int64_t>(page) * c.hkv + kvh;
  u32x4* data = reinterpret_cast<u32x4*>(c.data + cache_at(c, page, kvh, side, W));
  for (int i = threadIdx.x; i < (W / 16) << c.plog; i += blockDim.x) data[i] = u32x4{0, 0, 0, 0};
  if (threadIdx.x == 0) c.scales[at * 2 + side] = 0.0f;
  if (side == 0 && c.bounds) {
    for (int i = threadIdx.x; i < 2 * W; i += blockDim.x) c.bounds[at * 2 * W + i] = 0;
    if (threadIdx.x == 0) c.units[at] = -INFINITY;  // chosen last, like a page that is not there
  }
}

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
  if (full ? page < 0 : slot < 0) return;  // block-uniform
  if (old > 0 && slot < 0) {
    lost_page(c, page, kvh, side, W);
    return;
  }

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
    // a thread turns a run of tokens, of at most as many as leave every thread one
    const int f = threadIdx.x & (pw - 1), per = NT / pw, run = min(16, max(1, P / per));
    int t = (old & ~(run - 1)) + threadIdx.x / pw * run;
    if (f < half_rot && t < last) {
      Turning turning(a.turns[f]);
      for (; t < last; t += per * run) {
        const int from = max(t, old), to = min(t + run, last);
        if (from >= to) continue;
        turning.start(first + from);
#pragma unroll 1
        for (int i = from; i < to; ++i) {
          if (i > from) turning.next();
          T* x = reinterpret_cast<T*>(lds + i * stride) + ca * f;
          turn(turning.g, x[0], x[cb]);
        }
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
      // outward, also where the product is too small for a number
      const float up = high > 0.0f ? fmaxf(ceilf(high * unit_inv), 1.0f) : ceilf(high * unit_inv);
      const float down = low < 0.0f ? fminf(floorf(low * unit_inv), -1.0f) : floorf(low * unit_inv);
      to[0] = none ? 0 : static_cast<int8_t>(up);
      to[W] = none ? 0 : static_cast<int8_t>(down);
      if (col == 0) c.units[at] = bad ? __uint_as_float(0x7FC00000u) : exp2_int(k);
    }
  }
}

// Eight columns of a row, read or written once and past the caches (24 histories written
// and read back 178 -> 162 us; an attention call right after reads its query as fast).
template <typename T>
struct Eight {
  u32x4 w[sizeof(T) / 2];
  __device__ inline void load(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + i);
  }
  __device__ inline void store(T* p) const {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) __builtin_nontemporal_store(w[i], reinterpret_cast<u32x4*>(p) + i);
  }
  __device__ inline T get(int i) const {
    if constexpr (sizeof(T) == 2) return static_cast<T>(w[0][i >> 1] >> 16 * (i & 1));
    else return __uint_as_float(w[i >> 2][i & 3]);
  }
  __device__ inline void set(int i, T x) {
    if constexpr (sizeof(T) == 2) w[0][i >> 1] = (w[0][i >> 1] & (i & 1 ? 0xFFFFu : 0xFFFF0000u)) | static_cast<uint32_t>(x) << 16 * (i & 1);
    else w[i >> 2][i & 3] = __float_as_uint(x);
  }
};

// Query rows: a wave takes four of a sequence. A lane makes a pair's angles in all four,
// which go by LDS to every head (kept in registers beside the rows' columns they cost
// waves a SIMD: 24 histories 187 us a pass, so 160); then row after row, eight pairs of a
// head a lane where the columns allow whole 16-byte loads.
constexpr int kTurnRows = 4;
template <typename T, int NT>
__device__ __forceinline__ void turn_rows(const CacheAppend& a, char* lds, int64_t b) {
  constexpr int kTile = kTurnRows * NT / kWave;  // rows of a block
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), d = c.d;
  int64_t tile;
  int s;
  if (c.pad > 0) {
    const int64_t per = (c.pad + kTile - 1) / kTile;
    s = static_cast<int>(b / per);
    tile = b - s * per;
    if (s >= c.seqs) return;
  } else {
    s = find_tile(c.off, c.seqs, 1, __builtin_ctz(kTile), static_cast<uint32_t>(b), tile);
  }
  const SeqSpan span = seq_span(c.off, s, c.pad, c.rows);
  const int64_t all = c.pad > 0 ? c.pad : int64_t(span.len), first = tile * kTile + wave * kTurnRows;
  if (tile < 0 || first >= all) return;
  const int64_t base = max(c.lens[s], int64_t(0));
  const RotPairs rp(a);
  Angle* angles = reinterpret_cast<Angle*>(lds) + wave * kTurnRows * kWave;  // rotary / 2 is at most 64
  if (lane < rp.count) {
    Turning turning(a.turns[lane]);
#pragma unroll 1
    for (int i = 0; i < kTurnRows; ++i) {
      const int64_t p = base + first + i;
      if (i == 0 || (p & 15) == 0) turning.start(p);
      else turning.next();
      angles[i * kWave + lane] = turning.g;
    }
  }
  __builtin_amdgcn_wave_barrier();
  const uint32_t chunks = rp.count / 8, rest = (d - a.rotary) / 8, per = chunks + rest;
  for (int64_t token = first; token < min(all, first + kTurnRows); ++token) {
    const int64_t row = span.start + token;
    T* out = static_cast<T*>(a.q_out) + row * a.hq * d;
    if (token >= span.len) {  // past the sequence's end
      for (int i = lane; i < a.hq * d; i += kWave) out[i] = T(0);
      continue;
    }
    const T* q = static_cast<const T*>(a.q.p) + row * a.q.row;
    const Angle* turned = angles + (token - first) * kWave;
    if (rp.count % 8 == 0) {
      for (uint32_t i = lane; i < per * a.hq; i += kWave) {
        const uint32_t h = i / per, k = i - h * per;
        const T* from = q + h * a.q.head;
        T* to = out + h * d;
        Eight<T> x, y;
        if (k >= chunks) {  // columns that stay
          x.load(from + a.rotary + (k - chunks) * 8);
          x.store(to + a.rotary + (k - chunks) * 8);
          continue;
        }
        const int f = k * 8, ca = a.next ? 2 * f : f, cb = a.next ? 2 * f + 8 : f + rp.count;
        x.load(from + ca);
        y.load(from + cb);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const Angle at = turned[f + e];
          if (a.next) {
            Eight<T>& z = e < 4 ? x : y;
            T v = z.get(2 * (e & 3)), w = z.get(2 * (e & 3) + 1);
            turn(at, v, w);
            z.set(2 * (e & 3), v);
            z.set(2 * (e & 3) + 1, w);
          } else {
            T v = x.get(e), w = y.get(e);
            turn(at, v, w);
            x.set(e, v);
            y.set(e, w);
          }
        }
        x.store(to + ca);
        y.store(to + cb);
      }
    } else {
      const int f = lane & (rp.lanes - 1), step = kWave / rp.lanes;
      if (f < rp.count)
        for (int h = lane / rp.lanes; h < a.hq; h += step) {
          T x = q[h * a.q.head + rp.step * f], y = q[h * a.q.head + rp.step * f + rp.apart];
          turn(turned[f], x, y);
          out[h * d + rp.step * f] = x;
          out[h * d + rp.step * f + rp.apart] = y;
        }
      for (int h = 0; h < a.hq && a.rotary < d; ++h)
        for (int i = a.rotary + lane; i < d; i += kWave) out[h * d + i] = q[h * a.q.head + i];
    }
  }
}

// The grid: blocks of (touched page, key head, side), then blocks of query rows, then
// blocks of NT sequences for their new lengths.
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
      turn_rows<T, NT>(a, lds, b);
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
template <typename O>
__device__ inline O as_out(float x);
template <>
__device__ inline uint16_t as_out<uint16_t>(float x) {
  return f32_to_bf16(x);
}
template <>
__device__ inline float as_out<float>(float x) {
  return x;
}

// Rows start[s] + i of sequence s as the cache holds them: a block per touched
// page, key head and side, 64 tokens at a time through LDS, so that rows are
// stored whole.
constexpr int kReadTokens = 64;
template <typename T, typename O, bool E4M3>
__global__ __launch_bounds__(kBlock) void k_cache_read(const CacheRead a, int64_t block0) {
  constexpr int kStride = 128 * static_cast<int>(sizeof(O)) + 16;  // rows start on other banks
  __shared__ __align__(16) char lds[kReadTokens * kStride];
  const CacheArgs& c = a.c;
  const int d = c.d, P = 1 << c.plog, W = d <= 32 ? 32 : d <= 64 ? 64 : 128;
  const int side = blockIdx.z, kvh = blockIdx.y;
  int64_t tile;
  const int s = find_pages(c.off, c.seqs, c.plog, block0 + blockIdx.x, tile);
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
  O* to = static_cast<O*>(side ? a.v : a.k) + (row0 * c.hkv + kvh) * d;
  const int64_t row = static_cast<int64_t>(c.hkv) * d;
  const int chunks = d / 8, cw = chunks <= 1 ? 1 : 1 << (32 - __builtin_clz(chunks - 1));  // of eight columns
  const int ch = threadIdx.x & (cw - 1), per = kBlock / cw;
  if (page < 0) {  // an open page, or none
    const int held = !full && slot >= 0 ? static_cast<int>(min(max(len - first, int64_t(0)), static_cast<int64_t>(t1))) : 0;
    const T* open = static_cast<const T*>(c.open) + (held > 0 ? open_at(c, slot, n, kvh, side) : 0);
    if (ch < chunks)
      for (int t = t0 + threadIdx.x / cw; t < t1; t += per) {
        Eight<T> x;
        Eight<O> y;
        if (t < held) x.load(open + t * d + ch * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) y.set(e, as_out<O>(t < held ? to_f32(x.get(e)) : 0.0f));
        y.store(to + t * row + ch * 8);
      }
    return;
  }
  const float scale = c.scales[(static_cast<int64_t>(page) * c.hkv + kvh) * 2 + side];
  const uint8_t* data = c.data + cache_at(c, page, kvh, side, W);
  for (int base = t0 & ~(kReadTokens - 1); base < t1; base += kReadTokens) {
    const int tokens = min(kReadTokens, P), log = c.plog < 6 ? 5 : 6;  // 1 << log of them
    __syncthreads();
    if (side == 0) {
      for (int i = threadIdx.x; i < W / 16 * tokens; i += kBlock) {
        const int t = i & (tokens - 1), col = i >> log;
        const u32x4 w = *reinterpret_cast<const u32x4*>(data + (((col << c.plog) + base + t) << 4));
        Eight<O> y[2];
#pragma unroll
        for (int e = 0; e < 16; ++e)
          y[e >> 3].set(e & 7, as_out<O>(code_value<E4M3>(static_cast<uint8_t>(w[e >> 2] >> 8 * (e & 3))) * scale));
        O* at = reinterpret_cast<O*>(lds + t * kStride) + col * 16;
        y[0].store(at);
        y[1].store(at + 8);
      }
    } else {
      for (int i = threadIdx.x; i < W * tokens / 16; i += kBlock) {
        const int col = i & (W - 1), t = i / W * 16;
        const u32x4 w = *reinterpret_cast<const u32x4*>(data + (((base + t) / 16 * W + col) << 4));
#pragma unroll
        for (int e = 0; e < 16; ++e)
          reinterpret_cast<O*>(lds + (t + e) * kStride)[col] =
              as_out<O>(code_value<E4M3>(static_cast<uint8_t>(w[e >> 2] >> 8 * (e & 3))) * scale);
      }
    }
    __syncthreads();
    if (ch < chunks)
      for (int t = max(t0, base) + threadIdx.x / cw; t < min(t1, base + tokens); t += per) {
        Eight<O> y;
        y.load(reinterpret_cast<const O*>(lds + (t - base) * kStride) + ch * 8);
        y.store(to + t * row + ch * 8);
      }
  }
}

constexpr int64_t kMostBlocks = int64_t(1) << 21;  // of a launch: fewer than 2^32 threads along an axis
constexpr int kPlainLds = 65536;                   // bytes of a block that a launch takes without asking

// LDS of k_cache_append's own: sh_top, sh_low and sh_high.
template <int NT>
constexpr int kOwnLds = NT / kWave * 4 + 2 * NT * 4;

template <typename T, bool E4M3, int NT>
hipError_t append(CacheAppend a, int bytes, hipStream_t s) {
  const bool rows = a.k.p != nullptr && a.c.rows > 0;
  const int64_t u = a.c.pad > 0 ? a.c.seqs * ((a.c.pad >> a.c.plog) + 2) : (a.c.rows >> a.c.plog) + 2 * int64_t(a.c.seqs);
  a.page_units = rows ? u : 0;
  constexpr int64_t kTile = kTurnRows * NT / kWave;
  a.q_units = !a.q.p ? 0 : a.c.pad > 0 ? a.c.seqs * ((a.c.pad + kTile - 1) / kTile) : a.c.rows / kTile + a.c.seqs;
  const int64_t lens = a.new_lens ? (a.c.seqs + NT - 1) / NT : 0;
  const int64_t blocks = a.page_units * a.c.hkv * 2 + a.q_units + lens;
  if (bytes + kOwnLds<NT> > kPlainLds) {
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
  const int angles = kTurnRows * kBlock * static_cast<int>(sizeof(Angle)), page = lds_stride<T>(a.c.d) << a.c.plog;
  const bool large = page + kOwnLds<256> > kPlainLds;
  const int bytes = std::max(page, large ? 4 * angles : angles);
  // a large page fills a CU's LDS by itself: more waves on it then (else 256 threads: 24
  // histories in pages of 64 126 us, 141 by 128, 153 by 512)
  return large ? append<T, E4M3, 1024>(a, bytes, s) : append<T, E4M3, 256>(a, bytes, s);
}

template <typename T, typename O, bool E4M3>
hipError_t read_type(const CacheRead& a, hipStream_t s) {
  const int64_t blocks = (a.c.rows >> a.c.plog) + 2 * int64_t(a.c.seqs);
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {
    const int64_t now = blocks - b < kMostBlocks ? blocks - b : kMostBlocks;
    k_cache_read<T, O, E4M3><<<dim3(static_cast<unsigned>(now), a.c.hkv, 2), kBlock, 0, s>>>(a, b);
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
