// Device helpers of the attention kernels (gfx950): sequence geometry, the
// LDS tile, and fragments of the 32x32 matrix instructions for both types.
//
// Fragments.  v_mfma_f32_32x32x16_bf16 takes from lane l (half h = l / 32)
// eight consecutive k of row l % 32 of A (column l % 32 of B) and leaves in
// register r of lane l the element of row (r / 4) * 8 + h * 4 + r % 4, column
// l % 32.  fp32 uses v_mfma_f32_32x32x2_f32 eight times on the same eight
// values per lane: step e multiplies the k that both operands hold in slot e,
// so both types share one layout.
//
// The products are arranged so that a tile of probabilities never leaves its
// registers: the first product is taken with the long axis (keys in the
// forward, query rows in the gradient of k and v) along the rows, so a lane
// holds one column and 16 of its 32 rows; registers 8 t .. 8 t + 7 are then
// exactly slot 0 .. 7 of the next product's B operand, with slot e of half h
// standing for row 16 t + (e / 4) * 8 + h * 4 + e % 4.  The A operand (v, k,
// q or dout, transposed) is read from LDS in that order of its rows.
#pragma once

#include "device_common.h"
#include "seq_internal.h"

#pragma clang fp contract(fast)

namespace rs {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kAttnWaves = 4;
constexpr int kAttnRows = 32 * kAttnWaves;  // rows of a block's own tile: 32 per wave
constexpr int kAttnStep = 64;               // rows of the tile it walks over, per step

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct f32x8s {
  float v[8];
};

template <typename T>
struct Frag;
template <>
struct Frag<uint16_t> {
  typedef bf16x8 type;
};
template <>
struct Frag<float> {
  typedef f32x8s type;
};

__device__ inline f32x16 mma(const bf16x8& a, const bf16x8& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mma(const f32x8s& a, const f32x8s& b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}

// Two floats to bf16 (round to nearest even), in one word.
__device__ inline uint32_t pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Registers 8 t .. 8 t + 7 of a product as a B operand.  bf16: the
// probabilities (or their gradients) are rounded to 8 bits of mantissa here,
// once, as the matrix instruction takes them; their sum is kept in fp32.
template <typename T>
__device__ inline typename Frag<T>::type to_frag(const float (&p)[16], int t);
template <>
__device__ inline bf16x8 to_frag<uint16_t>(const float (&p)[16], int t) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16(p[8 * t + 2 * e], p[8 * t + 2 * e + 1]);
  return __builtin_bit_cast(bf16x8, w);
}
template <>
__device__ inline f32x8s to_frag<float>(const float (&p)[16], int t) {
  f32x8s f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = p[8 * t + e];
  return f;
}

template <typename T>
__device__ inline typename Frag<T>::type zero_frag();
template <>
__device__ inline bf16x8 zero_frag<uint16_t>() {
  return bf16x8{};
}
template <>
__device__ inline f32x8s zero_frag<float>() {
  return f32x8s{};
}

// Eight consecutive elements of global memory (16-byte aligned).
__device__ inline void load_frag(const uint16_t* p, bf16x8& f) { f = *reinterpret_cast<const bf16x8*>(p); }
__device__ inline void load_frag(const float* p, f32x8s& f) { f = *reinterpret_cast<const f32x8s*>(__builtin_assume_aligned(p, 16)); }

// A tile of rows of HD elements in LDS, in 16-byte chunks.  Chunk c of row r
// lies at chunk c ^ key(r) of its row, with the key chosen so that both reads
// spread over the 64 banks: 16 consecutive rows at one chunk (rows as an
// operand), and 4 consecutive rows times 64 bytes (rows transposed).
template <typename T, int HD>
struct Tile {
  static constexpr int kPer = 16 / sizeof(T);  // elements per chunk
  static constexpr int kChunks = HD / kPer;    // chunks per row
  static constexpr int kRowBytes = HD * sizeof(T);

  __device__ static inline int key(int r) {
    if (kChunks >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    if (kChunks == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return (r >> 2) & 3;
  }
  // Byte address of chunk c of row r.
  __device__ static inline int at(int r, int c) { return r * kRowBytes + ((c ^ key(r)) << 4); }
};

// Operand rows: elements k0 .. k0 + 7 (k0 = 16 t + 8 h) of row r.
template <int HD>
__device__ inline void row_frag(const char* tile, int r, int k0, bf16x8& f) {
  f = *reinterpret_cast<const bf16x8*>(tile + Tile<uint16_t, HD>::at(r, k0 >> 3));
}
template <int HD>
__device__ inline void row_frag(const char* tile, int r, int k0, f32x8s& f) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(tile + Tile<float, HD>::at(r, k0 >> 2));
  const f32x4 b = *reinterpret_cast<const f32x4*>(tile + Tile<float, HD>::at(r, (k0 >> 2) + 1));
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f.v[e] = a[e];
    f.v[4 + e] = b[e];
  }
}

// Transposed operand: for the 16 tile rows from r0, column c0 + l % 32, in the
// slot order described above.  bf16: ds_read_b64_tr_b16, where 16 lanes read
// four rows of 32 bytes (lane i the piece i % 4 of row i / 4) and lane i
// receives column i of the four rows.
template <int HD>
__device__ inline void col_frag(const char* tile, int r0, int c0, int lane, bf16x8& f) {
  const int r = r0 + (lane >> 5) * 4 + ((lane >> 2) & 3);
  const int c = c0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const char* p0 = tile + Tile<uint16_t, HD>::at(r, c >> 3) + (c & 7) * 2;
  const char* p1 = tile + Tile<uint16_t, HD>::at(r + 8, c >> 3) + (c & 7) * 2;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p0));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p1));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 ab = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  f = __builtin_bit_cast(bf16x8, ab);
}
template <int HD>
__device__ inline void col_frag(const char* tile, int r0, int c0, int lane, f32x8s& f) {
  const int c = c0 + (lane & 31), h = lane >> 5;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int r = r0 + (e >> 2) * 8 + h * 4 + (e & 3);
    f.v[e] = *reinterpret_cast<const float*>(tile + Tile<float, HD>::at(r, c >> 2) + (c & 3) * 4);
  }
}

// Where the distances |p - j| of a tile all have one sign, the distance term is
// linear in j and needs one operation with the register's constant instead of
// three: +1 if every key lies at or before every position, -1 if at or after.
__device__ inline int dist_sign(int first_key, int last_key, int least_pos, int most_pos) {
  return last_key <= least_pos ? 1 : first_key >= most_pos ? -1 : 0;
}

// The value of the lane's column in the other half of the wave.
__device__ inline float other_half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float other_half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// x = tanh(scale x) of 16 scores.  fp32 has the library's function.  bf16, by
// |scale x|: up to 1/2, x + x^3 P(x^2) with P fitted to the least largest error,
// off by 7e-8 of the value; above, 1 - 2 / (e^2x + 1) on the hardware's exp2 and
// reciprocal, off by 1e-7.  A score's value goes by itself alone, so that the
// passes agree on it; a wave whose scores are all small, as caps are used,
// leaves out the exponents.
template <typename T>
__device__ inline void tanh_scores(float (&x)[16], float scale);
template <>
__device__ inline void tanh_scores<float>(float (&x)[16], float scale) {
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = tanhf(x[i] * scale);
}
__device__ inline float tanh_small(float x) {
  const float u = x * x;
  const float p = -0.3333314955f + u * (0.1332598776f + u * (-0.0530529357f + u * 0.0172569603f));
  return x + x * (u * p);
}
template <>
__device__ inline void tanh_scores<uint16_t>(float (&x)[16], float scale) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] *= scale;
    most = fmaxf(most, fabsf(x[i]));
  }
  if (__all(most <= 0.5f)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = tanh_small(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float big = 1.0f - 2.0f * __builtin_amdgcn_rcpf(exp2_hw(x[i] * (2.0f * kLog2e)) + 1.0f);
      x[i] = fabsf(x[i]) <= 0.5f ? tanh_small(x[i]) : big;
    }
  }
}

// First row and length of sequence s among `rows` rows: packed, rows
// [off[s], off[s + 1]); padded, the first min(length, pad) rows of its block.
// Offsets outside the tensor are cut to it, so no access leaves it.
struct SeqSpan {
  int64_t start;
  int len;
};
__device__ inline SeqSpan seq_span(const int64_t* __restrict__ off, int s, int64_t pad, int64_t rows) {
  const int64_t o = off[s];
  int64_t len = off[s + 1] - o;
  SeqSpan r;
  if (pad > 0) {
    r.start = s * pad;
    len = min(len, pad);
  } else {
    r.start = min(max(o, int64_t(0)), rows);
    len = min(len, rows - r.start);
  }
  r.len = static_cast<int>(max(len, int64_t(0)));
  return r;
}

// Block numbers over ragged sequences without a table: sequence s owns the
// numbers from off[s] * mul / per + s on.  They are enough for
// ceil(len * mul / per) tiles (floor((o + n) / per) - floor(o / per) + 1 >=
// ceil(n / per)), strictly increasing in s, and end below
// off[seqs] * mul / per + seqs.  Returns the sequence of block b, found by the
// wave in steps of 64 sequences at a time, and the tile inside it: below 0 for
// a block before the first sequence (off[0] > 0, or offsets that fall).
__device__ inline int64_t tile_base(const int64_t* __restrict__ off, int s, int mul, int per) {
  return max(off[s], int64_t(0)) * mul / per + s;
}
__device__ inline int find_seq(const int64_t* __restrict__ off, int seqs, int mul, int per, int64_t b, int64_t& tile) {
  const int lane = threadIdx.x & (kWave - 1);
  int lo = 0, n = seqs;
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave;
    const int s = lane * step;
    const bool below = s < n && tile_base(off, lo + s, mul, per) <= b;
    const int c = max(1, static_cast<int>(__popcll(__ballot(below))));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  tile = b - tile_base(off, lo, mul, per);
  return lo;
}

// r / group; most models have one query head per key head, or a power of two.
__device__ inline int div_group(int r, int group) {
  if ((group & (group - 1)) == 0) return r >> (31 - __builtin_clz(group));  // uniform
  return r / group;
}

// A one-dimensional grid of tiles times key heads.  Neighbouring tiles read the
// same keys (or rows), so runs of kTileRun consecutive tiles of one key head go
// to one XCD and its L2; `back` takes the tiles from the last, which see the
// most keys under a causal mask, to the first, so that the short ones fill in
// at the end.
constexpr uint32_t kTileRun = 8;
struct BlockOf {
  int64_t tile;
  int kvh;
};
__device__ inline BlockOf block_of(const AttnArgs& a, bool back) {
  const uint32_t tiles = a.blocks / a.hkv;
  uint32_t b = xcd_runs<kTileRun>(a.block0 + blockIdx.x, a.blocks);
  if (back) b = a.blocks - 1 - b;
  BlockOf x;
  x.kvh = b / tiles;
  x.tile = b - x.kvh * tiles;
  return x;
}

// The kernel over so many blocks, in launches of at most 2^22 of them, whole sets
// of tile runs.
template <int THREADS, typename K>
inline void launch_blocks(K* kernel, AttnArgs a, int64_t blocks, hipStream_t s) {
  constexpr int64_t kMost = int64_t(1) << 22;
  static_assert(kMost * THREADS < int64_t(1) << 32 && kMost % (8 * kTileRun) == 0, "a launch's threads");
  a.blocks = static_cast<uint32_t>(blocks);
  for (int64_t b = 0; b < blocks; b += kMost) {
    a.block0 = static_cast<uint32_t>(b);
    kernel<<<static_cast<unsigned>(blocks - b < kMost ? blocks - b : kMost), THREADS, 0, s>>>(a);
  }
}

// Rows of a sequence are packed head by head: row r is token r / group, query
// head kvh * group + r % group, so that the query heads of a key head share
// its tiles.  Row r sees the keys j < limit.
struct RowOf {
  int token, head;
};
__device__ inline RowOf row_of(int r, int kvh, int group) {
  RowOf x;
  x.token = div_group(r, group);
  x.head = kvh * group + (r - x.token * group);
  return x;
}
__device__ inline int key_limit(int token, int lq, int lk, bool causal, int prefix) {
  if (!causal) return lk;
  return min(lk, max(token + lk - lq + 1, prefix));
}

// Rows of a [rows][heads][d] tensor to an LDS tile of N rows, by loads
// that write LDS themselves (16 bytes per lane, a wave's 1 KiB back to back):
// no registers hold them and the wave goes on; wait_tiles() before their use.
// The lane picks the chunk that belongs at its place, so the tile's chunk
// order costs nothing.  The buffer's bounds do the masking: rows past the
// sequence's end and columns past d lie outside and arrive as zeros.  A wave's
// rows are consecutive (at most 32) and its buffer starts at the first of them:
// their offsets stay below 2^31, where the bounds end, up to the largest stride.
template <typename T, int HD, int N = kAttnStep, int W = kAttnWaves>
struct TileLoader {
  typedef Tile<T, HD> L;
  static constexpr int kLoads = N * L::kRowBytes / (W * kWave * 16);  // per thread of W waves
  static_assert(kLoads >= 1 && kLoads * W * kWave * 16 == N * L::kRowBytes, "whole loads");
  static constexpr int kRows = N / W;  // a wave's share
  static_assert(kRows * W == N && kRows <= 32, "32 rows of 2^23 fp32 elements span 2^30 bytes");
  uint32_t off[kLoads];  // byte offset of the thread's chunks from the wave's first row
  int64_t row_bytes;
  const char* base;  // the wave's first row of the sequence's first tile
  int len, d_bytes;  // rows from there to the sequence's end

  __device__ inline void init(const void* p, int64_t start, int64_t row, int64_t head_off, int d, int n) {
    const int wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1);
    row_bytes = row * static_cast<int64_t>(sizeof(T));
    base = static_cast<const char*>(p) + ((start + wave * kRows) * row + head_off) * static_cast<int64_t>(sizeof(T));
    len = n - wave * kRows;
    d_bytes = d * static_cast<int>(sizeof(T));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = (i * kWave + lane) * 16;
      const int r = at / L::kRowBytes, c = ((at % L::kRowBytes) >> 4) ^ L::key(wave * kRows + r);
      off[i] = c * 16 < d_bytes ? r * static_cast<uint32_t>(row_bytes) + c * 16 : 0x80000000u;
    }
  }
  // Rows j0 .. j0 + N - 1 of the sequence (j0 < its length).
  __device__ inline void load(char* tile, int j0) const {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass has no buffer descriptors
    const int rows = min(kRows, len - j0);
    const int bytes = rows > 0 ? (rows - 1) * static_cast<int>(row_bytes) + d_bytes : 0;
    const char* p = base + j0 * row_bytes;
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    // readfirstlane gives a signed int: no sign may reach the upper word
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(static_cast<uint64_t>(hi) << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes),
        0x00020000);
    char* dst = tile + (W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * kLoads * kWave * 16);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc, (__attribute__((address_space(3))) void*)(dst + i * kWave * 16), 16, off[i], 0, 0, 0);
#endif
  }
};

// The same for packed query rows, a step of N rows of whole tokens: floor(N /
// group) tokens with all their heads, or where a group has more than N heads,
// N of one token's.  The offsets inside a step never change; rows past the step's
// tokens or the sequence's end are sent out of the buffer's bounds.
template <int N>
struct RowSteps {
  int tokens, parts;  // tokens per step, steps per token (one of them is 1)
  __device__ inline explicit RowSteps(int g) : tokens(g <= N ? N / g : 1), parts(g <= N ? 1 : (g + N - 1) / N) {}
};
template <typename T, int HD, int N, int W>
struct RowLoader {
  typedef Tile<T, HD> L;
  static constexpr int kLoads = N * L::kRowBytes / (W * kWave * 16);
  static_assert(kLoads >= 1 && kLoads * W * kWave * 16 == N * L::kRowBytes, "whole loads");
  static constexpr int kRows = N / W;  // a wave's share
  static_assert(kRows * W == N && kRows <= 16, "at most 16 tokens and a group of heads: below 2^31 bytes");
  uint32_t off[kLoads];
  int64_t row_bytes, head_bytes;
  const char* base;  // the sequence's first token (of the wave's rows), the group's first head

  __device__ inline void init(const HeadRows& t, int64_t start, int kvh, int group, int d) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1);
    const int tok0 = group <= N ? div_group(wave * kRows, group) : 0;  // of the wave's first row
    row_bytes = t.row * static_cast<int64_t>(sizeof(T));
    head_bytes = t.head * static_cast<int64_t>(sizeof(T));
    base = static_cast<const char*>(t.p) + (start + tok0) * row_bytes + static_cast<int64_t>(kvh) * group * head_bytes;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = ((wave * kLoads + i) * kWave + lane) * 16;
      const int r = at / L::kRowBytes, c = ((at % L::kRowBytes) >> 4) ^ L::key(r);
      const int tok = group <= N ? div_group(r, group) : 0;
      off[i] = c * 16 < d * static_cast<int>(sizeof(T))
                   ? (tok - tok0) * static_cast<uint32_t>(row_bytes) +
                         (r - tok * group) * static_cast<uint32_t>(head_bytes) + c * 16
                   : 0x80000000u;
    }
  }
  // The step from token `tok`, head `head` of the group; `count` rows of it exist.
  __device__ inline void load(char* tile, int tok, int head, int count) const {
#if defined(__HIP_DEVICE_COMPILE__)
    const char* p = base + tok * row_bytes + head * head_bytes;
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(static_cast<uint64_t>(hi) << 32 | lo), 0, 0x7FFFFFFF, 0x00020000);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1);
    char* dst = tile + wave * kLoads * kWave * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = ((wave * kLoads + i) * kWave + lane) * 16 / L::kRowBytes;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc, (__attribute__((address_space(3))) void*)(dst + i * kWave * 16), 16, r < count ? off[i] : 0x80000000u, 0,
          0, 0);
    }
#endif
  }
};

// All but the wave's last N loads have arrived.
template <int N>
__device__ inline void wait_loads() {
  static_assert(N < 64, "the counter has six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4 | 15 << 8);
}

// Every load of the wave has arrived, and then every wave's.
__device__ inline void wait_tiles() {
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
}

// What rounding to bf16 takes away from x.
__device__ inline float rest_bf16(float x) {
  return x - __uint_as_float(pack_bf16(x, 0.0f) << 16);
}

// Four consecutive elements of an output row from registers 4 i .. 4 i + 3.
__device__ inline void store4(uint16_t* p, float a, float b, float c, float d) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}
__device__ inline void store4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}

// A wave's 32 output rows, one per lane column, through LDS: a lane holds four
// elements of a row at a time, and storing them as they lie would send 32
// requests of 16 bytes per instruction to L2 (half the time of the forward on
// sequences of 560 keys of 64); from LDS, consecutive lanes store whole rows.
template <typename T, int HD>
struct RowWriter {
  static constexpr int kStride = HD * sizeof(T) + 16;  // rows start on other banks
  static constexpr int kBytes = 32 * kStride;
  // value(i, e): the lane's element of register e (0 .. 15) of column tile i
  template <typename V>
  __device__ static inline void put(char* region, int lane, V value) {
    char* row = region + (lane & 31) * kStride + (lane >> 5) * 4 * sizeof(T);
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store4(reinterpret_cast<T*>(row) + i * 32 + g * 8, value(i, 4 * g), value(i, 4 * g + 1), value(i, 4 * g + 2),
               value(i, 4 * g + 3));
  }
  // at(row): where row 0 .. 31 goes, or null
  template <typename A>
  __device__ static inline void flush(const char* region, int lane, int d, A at) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int kPer = 16 / sizeof(T), kChunks = HD / kPer;
#pragma unroll
    for (int n = 0; n < 32 * kChunks / kWave; ++n) {
      const int idx = n * kWave + lane, r = idx / kChunks, c = idx % kChunks;
      T* p = at(r);
      if (p && c * kPer < d)
        *reinterpret_cast<u32x4*>(p + c * kPer) = *reinterpret_cast<const u32x4*>(region + r * kStride + c * 16);
    }
  }
};

}  // namespace rs
