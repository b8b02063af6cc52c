// The pages of a sequence that a query looks at: a cheap score of every full
// page from the bounds of its keys' columns, and the highest `count` of them
// (gfx950).
//
//   q8 = rne(q / sq), sq the least power of two with max |q| <= 127 sq
//   I  = sum_c max(q8_c mx_c, q8_c mn_c) = sum_c q8+_c mx_c + q8-_c mn_c
//   score(page) = unit max_h (sq_h I_h) over the query heads of the key head
//
// mx and mn bound the page's keys column by column, so with q8 for q a score is
// not below that of any key in the page. Everything is whole numbers of at most
// 8 bits and powers of two: I is below 2^24, the products are exact, and the
// choice does not depend on the order of any sum. Equal scores go to the lower
// page.
//
// A thread takes one page, its bounds in registers, against every head; the
// query's words are the same for all lanes and come from LDS.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_common.h"

namespace rs {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kHeadsAtOnce = 16;

__device__ inline float to_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ inline float to_f32(float x) { return x; }

// The sequence of a row, by the wave, and the row's place in it; false for a row
// outside every sequence.
struct RowAt {
  int s, token, len, lk;
};
__device__ inline bool row_at(const CacheArgs& c, int64_t row, RowAt& x) {
  int64_t token;
  if (c.pad > 0) {
    x.s = static_cast<int>(row / c.pad);
    token = row - x.s * c.pad;
  } else {
    const int lane = threadIdx.x & (kWave - 1);
    int lo = 0, n = c.seqs;
    while (n > 1) {
      const int step = (n + kWave - 1) / kWave;
      const int s = lane * step;
      const bool below = s < n && c.off[lo + s] <= row;
      const int k = max(1, static_cast<int>(__popcll(__ballot(below))));
      lo += (k - 1) * step;
      n = min(step, n - (k - 1) * step);
    }
    x.s = __builtin_amdgcn_readfirstlane(lo);
    token = row - c.off[x.s];
  }
  const SeqSpan q = seq_span(c.off, x.s, c.pad, c.rows);
  if (token < 0 || token >= q.len) return false;
  x.token = static_cast<int>(token);
  x.len = q.len;
  x.lk = cache_len(c, x.s);
  return true;
}
// Full pages that the query sees anything of.
__device__ inline int pages_seen(const CacheSelect& a, const RowAt& x) {
  const int n = x.lk >> a.c.plog;
  if (!a.causal) return n;
  const int pos = x.token + x.lk - x.len;
  return pos < 0 ? 0 : min(n, (pos >> a.c.plog) + 1);
}

// Grid: rows of the launch times a.tiles runs of 256 pages, key heads.
template <typename T, int W>
__global__ __launch_bounds__(kBlock) void k_select_score(const CacheSelect a) {
  constexpr int kWords = 2 * W / 4;
  __shared__ __align__(16) uint32_t q8[kHeadsAtOnce][kWords];
  __shared__ float sq[kHeadsAtOnce];
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t at_row = blockIdx.x / a.tiles, row = a.row0 + at_row;
  const int kvh = blockIdx.y;
  RowAt x;
  if (!row_at(c, row, x)) return;  // block-uniform, as below
  const int seen = pages_seen(a, x);
  if (seen <= a.count) return;  // all of them
  for (int page0 = (blockIdx.x - static_cast<uint32_t>(at_row) * a.tiles) * kBlock; page0 < seen; page0 += a.tiles * kBlock) {
    const int n = page0 + threadIdx.x;
    const int page = n < seen ? cache_page(c, x.s, n) : -1;
    u32x4 box[kWords / 4];
    float unit = 0.0f;
  #pragma unroll
    for (int i = 0; i < kWords / 4; ++i) box[i] = u32x4{0, 0, 0, 0};
    if (page >= 0) {
      const int64_t at = static_cast<int64_t>(page) * c.hkv + kvh;
      const u32x4* p = reinterpret_cast<const u32x4*>(c.bounds + at * 2 * W);
  #pragma unroll
      for (int i = 0; i < kWords / 4; ++i) box[i] = p[i];
      unit = c.units[at];
    }
    float best = -INFINITY;
    for (int h0 = 0; h0 < a.group; h0 += kHeadsAtOnce) {
      const int heads = min(kHeadsAtOnce, a.group - h0);
      __syncthreads();
      for (int h = wave; h < heads; h += kBlock / kWave) {
        const T* q = static_cast<const T*>(a.q.p) + row * a.q.row + static_cast<int64_t>(kvh * a.group + h0 + h) * a.q.head;
        float v[2];
        uint32_t top = 0;
  #pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int col = i * kWave + lane;
          v[i] = col < c.d ? to_f32(q[col]) : 0.0f;
          top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
  #pragma unroll
        for (int i = kWave / 2; i > 0; i >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), i, kWave)));
        const bool bad = top >= 0x7F800000u;  // a query that is not finite finds every page alike
        const int k = bad ? 0 : unit_exp(__uint_as_float(top), 1.984375f, 6);
        const float inv = exp2_int(-k);
        int8_t* to = reinterpret_cast<int8_t*>(q8[h]);
  #pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int col = i * kWave + lane;
          if (col >= W) continue;
          const int w = bad ? 0 : static_cast<int>(rintf(v[i] * inv));
          to[col] = static_cast<int8_t>(max(w, 0));
          to[W + col] = static_cast<int8_t>(min(w, 0));
        }
        if (lane == 0) sq[h] = exp2_int(k);
      }
      __syncthreads();
      for (int h = 0; h < heads; ++h) {
        int sum = 0;
  #pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(&q8[h][4 * i]);
  #pragma unroll
          for (int e = 0; e < 4; ++e)
            sum = __builtin_amdgcn_sdot4(static_cast<int>(box[i][e]), static_cast<int>(w[e]), sum, false);
        }
        best = fmaxf(best, static_cast<float>(sum) * sq[h]);
      }
    }
    float y = best * unit + 0.0f;  // one zero
    if (y != y) y = INFINITY;      // a page that is not finite is looked at
    if (page < 0) y = -INFINITY;   // one that is not there last of all
    if (n < seen) a.scores[(at_row * c.hkv + kvh) * c.width + n] = y;
  }
}

// Larger scores have larger keys.
__device__ inline uint32_t order(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A block per row and key head: the count-th largest key byte by byte from the
// top, by histograms, then the pages above it and the first of those equal to it.
template <int NT>
__global__ __launch_bounds__(NT) void k_select_pick(const CacheSelect a) {
  __shared__ int hist[256];
  __shared__ int sh[NT / kWave + 1];
  __shared__ uint32_t sh_prefix;
  __shared__ int sh_left;
  const CacheArgs& c = a.c;
  const int64_t row = a.row0 + blockIdx.x;
  const int kvh = blockIdx.y;
  int32_t* out = a.out + (row * c.hkv + kvh) * a.count;
  RowAt x;
  if (!row_at(c, row, x)) {
    // rows outside every sequence stay as they are; those of the padded copy name no page
    if (c.pad > 0)
      for (int i = threadIdx.x; i < a.count; i += NT) out[i] = -1;
    return;
  }
  const int seen = pages_seen(a, x);
  if (seen <= a.count) {
    for (int i = threadIdx.x; i < a.count; i += NT) out[i] = i < seen ? i : -1;
    return;
  }
  const float* score = a.scores + (static_cast<int64_t>(blockIdx.x) * c.hkv + kvh) * c.width;
  uint32_t prefix = 0;
  int left = a.count;  // still to be found among the keys with this prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += NT) hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0 : 0xFFFFFFFFu << (shift + 8);
    for (int i = threadIdx.x; i < seen; i += NT) {
      const uint32_t k = order(score[i]);
      if ((k & mask) == prefix) atomicAdd(&hist[k >> shift & 255], 1);
    }
    __syncthreads();
    if (threadIdx.x < kWave) {  // one wave, four bins a lane, from the top
      int h[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = hist[255 - (threadIdx.x * 4 + i)];
        sum += h[i];
      }
      const int incl = wave_incl_scan(sum);
      int above = incl - sum;
      if (above < left && incl >= left) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < left && above + h[i] >= left) {
            sh_prefix = prefix | static_cast<uint32_t>(255 - (threadIdx.x * 4 + i)) << shift;
            sh_left = left - above;
          }
          above += h[i];
        }
      }
    }
    __syncthreads();
    prefix = sh_prefix;
    left = sh_left;
  }
  // a run of pages per thread: how many of them are above, how many equal
  const int per = (seen + NT - 1) / NT, i0 = threadIdx.x * per, i1 = min(i0 + per, seen);
  int above = 0, equal = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = order(score[i]);
    above += k > prefix;
    equal += k == prefix;
  }
  int total;
  const int equal_before = block_excl_scan<NT>(equal, sh, total);
  const int take = min(max(left - equal_before, 0), equal);
  int at = block_excl_scan<NT>(above + take, sh, total);
  int taken = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = order(score[i]);
    const bool mine = k > prefix || (k == prefix && taken < take);
    taken += k == prefix;
    if (mine) out[at++] = i;
  }
}

constexpr size_t kMostScoreBytes = size_t(256) << 20;

}  // namespace

size_t plan_cache_select(const CacheSelect& a, int64_t* tokens) {
  const size_t one = static_cast<size_t>(a.c.hkv) * std::max<int64_t>(a.c.width, 1) * sizeof(float);
  *tokens = 0;
  if (a.c.rows == 0 || a.c.seqs == 0) return 0;
  *tokens = std::min<int64_t>(a.c.rows, std::max<int64_t>(1, kMostScoreBytes / one));
  *tokens = std::min<int64_t>(*tokens, int64_t(1) << 22);
  return *tokens * one;
}

template <typename T, int W>
static void run_select(const CacheSelect& a, hipStream_t s) {
  // fewer than 2^32 threads: a launch's scores are at most 2^26 (or one row's)
  if (a.c.width > a.count)
    k_select_score<T, W><<<dim3(static_cast<unsigned>(a.tokens * a.tiles), a.c.hkv), kBlock, 0, s>>>(a);
  const dim3 rows(static_cast<unsigned>(a.tokens), a.c.hkv);
  if (a.tiles > 16) k_select_pick<1024><<<rows, 1024, 0, s>>>(a);
  else k_select_pick<256><<<rows, 256, 0, s>>>(a);
}

hipError_t launch_cache_select(CacheSelect a, bool bf16, hipStream_t s) {
  int64_t tokens;
  plan_cache_select(a, &tokens);
  // the bound of the lengths only shapes the launches: a block goes on to the pages past it
  const int64_t pages = a.max_pages > 0 ? std::min(a.max_pages, a.c.width) : a.c.width;
  a.tiles = static_cast<int>(std::max<int64_t>(1, (pages + kBlock - 1) / kBlock));
  const int W = cache_width(a.c.d);
  for (int64_t r = 0; r < a.c.rows && tokens > 0; r += tokens) {
    a.row0 = r;
    a.tokens = std::min(tokens, a.c.rows - r);
    if (bf16) W == 32 ? run_select<uint16_t, 32>(a, s) : W == 64 ? run_select<uint16_t, 64>(a, s) : run_select<uint16_t, 128>(a, s);
    else W == 32 ? run_select<float, 32>(a, s) : W == 64 ? run_select<float, 64>(a, s) : run_select<float, 128>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace rs
