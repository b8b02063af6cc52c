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
// The scores are a matrix product in 8-bit integers, query heads by pages, over
// the q8+ with the maxima and the q8- with the minima one after the other. A wave
// loads the bounds of 16 pages as the instruction takes them, 64 pages ahead.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_common.h"

namespace rs {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kPagesAtOnce = 64;  // of a wave
constexpr int kPageRun = kPagesAtOnce * (kBlock / kWave);

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

// Grid: runs of kPageRun pages, runs of a.run rows of the launch, key heads. Rows
// of one sequence share the pages' bounds: a tile of 16 is 4, 2 or 1 of them, as
// many heads as a key head has (to a multiple of 4), or 16 of a row's more heads.
template <typename T, int W>
__global__ __launch_bounds__(kBlock) void k_select_score(const CacheSelect a) {
  constexpr int kSteps = 2 * W / 64, kGroups = kPagesAtOnce / 16;
  constexpr int kStride = 2 * W + 16;  // bytes: rows start on other banks
  __shared__ __align__(16) char q8[16 * kStride];
  __shared__ float sq[16];
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane & 15, grp = lane >> 4;
  const int kvh = blockIdx.z;
  const int64_t row0 = a.row0 + static_cast<int64_t>(blockIdx.y) * a.run, row_end = min(row0 + a.run, a.row0 + a.tokens);
  const int slots = a.group <= 4 ? 4 : a.group <= 8 ? 8 : 16;  // rows of a tile that a query row takes
  i32x4 box[kGroups][kSteps];
  float unit[kGroups];
  for (int64_t row = row0; row < row_end;) {
    RowAt x;
    if (!row_at(c, row, x)) {  // block-uniform, as all below
      ++row;
      continue;
    }
    const int64_t left = min(row_end - row, static_cast<int64_t>(x.len - x.token));  // rows here of the sequence
    RowAt end = x;
    end.token = x.token + static_cast<int>(left) - 1;
    const int most = pages_seen(a, end);
    if (most <= a.count) {  // all of them
      row += left;
      continue;
    }
    for (int page0 = blockIdx.x * kPageRun; page0 < most; page0 += gridDim.x * kPageRun) {
      const int first = page0 + wave * kPagesAtOnce;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int n = first + i * 16 + col;
        const int page = n < most ? cache_page(c, x.s, n) : -1;
        const int64_t at = static_cast<int64_t>(max(page, 0)) * c.hkv + kvh;
        const int8_t* p = c.bounds + at * 2 * W + grp * 16;
        // one that is not there comes last of all
        unit[i] = -INFINITY;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) box[i][k] = i32x4{0, 0, 0, 0};
        if (page >= 0) {
          unit[i] = c.units[at];
#pragma unroll
          for (int k = 0; k < kSteps; ++k) box[i][k] = *reinterpret_cast<const i32x4*>(p + k * 64);
        }
      }
      for (int64_t r = row; r < row + left; r += 16 / slots) {
        float best[kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) best[i] = -INFINITY;
        for (int h0 = 0; h0 < a.group; h0 += 16) {
          __syncthreads();
          // a wave takes four of the tile's rows
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int at = wave * 4 + y, head = h0 + at % slots;
            const int64_t own = r + at / slots;
            const bool there = own < row + left && head < a.group;
            float v[2] = {0.0f, 0.0f};
            uint32_t top = 0;
            if (there) {
              const T* q = static_cast<const T*>(a.q.p) + own * a.q.row + static_cast<int64_t>(kvh * a.group + head) * a.q.head;
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int d = i * kWave + lane;
                if (d < c.d) v[i] = to_f32(q[d]);
                top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
              }
            }
#pragma unroll
            for (int i = kWave / 2; i > 0; i >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), i, kWave)));
            const bool bad = top >= 0x7F800000u;  // a query that is not finite finds every page alike
            const int k = bad ? 0 : unit_exp(__uint_as_float(top), 1.984375f, 6);
            const float inv = exp2_int(-k);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int d = i * kWave + lane;
              if (d >= W) continue;
              const int w = bad ? 0 : static_cast<int>(rintf(v[i] * inv));
              q8[at * kStride + d] = static_cast<char>(max(w, 0));
              q8[at * kStride + W + d] = static_cast<char>(min(w, 0));
            }
            if (lane == 0) sq[at] = there ? exp2_int(k) : -1.0f;
          }
          __syncthreads();
          i32x4 qa[kSteps];
#pragma unroll
          for (int k = 0; k < kSteps; ++k)
            qa[k] = *reinterpret_cast<const i32x4*>(q8 + col * kStride + k * 64 + grp * 16);
          float scale[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) scale[e] = sq[grp * 4 + e];
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            i32x4 sum = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < kSteps; ++k) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(qa[k], box[i][k], sum, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (scale[e] > 0.0f) best[i] = fmaxf(best[i], static_cast<float>(sum[e]) * scale[e]);
          }
        }
        const int own = grp * 4 / slots;  // the lane's row
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          float y = best[i];
          if (slots >= 8) y = fmaxf(y, __shfl_xor(y, 16, kWave));
          if (slots >= 16) y = fmaxf(y, __shfl_xor(y, 32, kWave));
          const float s = unit[i] == -INFINITY ? -INFINITY : y * unit[i] + 0.0f;  // one zero
          const int n = first + i * 16 + col;
          if (n < most && r + own < row + left && grp * 4 % slots == 0)
            a.scores[((r + own - a.row0) * c.hkv + kvh) * c.width + n] = s == s ? s : INFINITY;  // a page that is not finite comes first
        }
      }
    }
    __syncthreads();
    row += left;
  }
}

// Larger scores have larger keys.
__device__ inline uint32_t order(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A block per row and key head, its keys in registers: the count-th largest by
// halving the range of keys (a step is one compare a key and one barrier; scores
// that differ are told apart after about as many steps as the pages' number has
// bits, where histograms of their bytes put most of them into a few counters: 15,626
// pages 40 us by histograms), then the pages above it and the first of
// those equal to it, in order.
template <int NT, int ITEMS>
__global__ __launch_bounds__(NT) void k_select_pick(const CacheSelect a) {
  constexpr int kWaves = NT / kWave;
  __shared__ int count_of[2][kWaves];
  __shared__ uint32_t top_of[kWaves];
  __shared__ int before[ITEMS * kWaves];  // pages taken (or equal) in the chunks of each wave before
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
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
  uint32_t key[ITEMS];  // 0: no page (order gives no score 0)
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int n = i * NT + threadIdx.x;
    key[i] = n < seen ? order(score[n]) : 0;
    top = max(top, key[i]);
  }
#pragma unroll
  for (int i = kWave / 2; i > 0; i >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), i, kWave)));
  if (lane == 0) top_of[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) top = max(top, top_of[i]);
  // at least `count` keys are >= low, fewer are >= high; `above` of them
  uint32_t low = 1, high = top + 1;
  int above = 0, side = 0;
  while (high - low > 1) {
    const uint32_t mid = low + (high - low) / 2;
    int n = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) n += static_cast<int>(__popcll(__ballot(key[i] >= mid)));
    if (lane == 0) count_of[side][wave] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) n += count_of[side][i];
    side ^= 1;  // the next step's counts go where nobody reads any more
    if (n >= a.count) {
      low = mid;
      if (n == a.count) break;
    } else {
      high = mid;
      above = n;
    }
  }
  // the keys from `high` on, and of those in [low, high) the first count - above
  const uint64_t below = (uint64_t(1) << lane) - 1;
  // what the chunks before hold: `before` to running sums, by the first wave
  auto sums = [&]() {
    __syncthreads();
    if (wave == 0) {
      int run = 0;
      for (int i = 0; i < ITEMS * kWaves; i += kWave) {
        const int v = i + lane < ITEMS * kWaves ? before[i + lane] : 0, incl = wave_incl_scan(v);
        if (i + lane < ITEMS * kWaves) before[i + lane] = run + incl - v;
        run += __shfl(incl, kWave - 1, kWave);
      }
    }
    __syncthreads();
  };
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint64_t equal = __ballot(key[i] >= low && key[i] < high);
    if (lane == 0) before[i * kWaves + wave] = static_cast<int>(__popcll(equal));
  }
  sums();
  uint64_t take[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const bool equal = key[i] >= low && key[i] < high;
    const int rank = before[i * kWaves + wave] + static_cast<int>(__popcll(__ballot(equal) & below));
    take[i] = __ballot(key[i] >= high || (equal && rank < a.count - above));
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
    if (lane == 0) before[i * kWaves + wave] = static_cast<int>(__popcll(take[i]));
  sums();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
    if (take[i] >> lane & 1) out[before[i * kWaves + wave] + static_cast<int>(__popcll(take[i] & below))] = i * NT + threadIdx.x;
}

// The same for any number of pages, read again for each step: the count-th largest
// key byte by byte from the top, by histograms.
template <int NT>
__global__ __launch_bounds__(NT) void k_select_pick_any(const CacheSelect a) {
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
  *tokens = std::min<int64_t>(*tokens, 65535);  // rows of a launch: they lie along its second axis
  return *tokens * one;
}

template <typename T, int W>
static void run_select(const CacheSelect& a, hipStream_t s) {
  if (a.c.width > a.count) {
    const dim3 grid(a.tiles, static_cast<unsigned>((a.tokens + a.run - 1) / a.run), a.c.hkv);
    k_select_score<T, W><<<grid, kBlock, 0, s>>>(a);
  }
  const dim3 rows(static_cast<unsigned>(a.tokens), a.c.hkv);
  if (a.c.width <= 1024) k_select_pick<256, 4><<<rows, 256, 0, s>>>(a);
  else if (a.c.width <= 16384) k_select_pick<1024, 16><<<rows, 1024, 0, s>>>(a);
  else if (a.c.width <= 65536) k_select_pick<1024, 64><<<rows, 1024, 0, s>>>(a);
  else k_select_pick_any<1024><<<rows, 1024, 0, s>>>(a);
}

hipError_t launch_cache_select(CacheSelect a, bool bf16, hipStream_t s) {
  int64_t tokens;
  plan_cache_select(a, &tokens);
  // the bound of the lengths only shapes the launches: a block goes on to the pages past it
  const int64_t pages = a.max_pages > 0 ? std::min(a.max_pages, a.c.width) : a.c.width;
  a.tiles = static_cast<int>(std::min<int64_t>(1 << 20, std::max<int64_t>(1, (pages + kPageRun - 1) / kPageRun)));
  // rows that a block takes: about those of a sequence, at most 16
  a.run = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(16, a.c.rows / a.c.seqs)));
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
