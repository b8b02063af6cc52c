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
// 8 bits and powers of two: I has at most 21 bits (128 * 127 * 127), the products are
// exact, and the choice does not depend on the order of any sum. A score may pass the
// range of fp32 (2^-252 to 2^263), so it is taken in 64 bits and kept as the upper
// half of those, which holds it all. Equal scores go to the lower page.
//
// The scores are a matrix product in 8-bit integers, query heads by pages, over
// the q8+ with the maxima and the q8- with the minima one after the other. A wave
// loads the bounds of 16 pages as the instruction takes them, 64 pages ahead, and
// the queries become bytes in LDS meanwhile, once for a tile of a sequence's rows.
// (Dot products of 4 bytes, a thread a page: 4 rows of 32 heads over 15,625 pages
// of 8 key heads 27 us; as matrices 13 to 14, the 33 MB of bounds at 2.4 TB/s: bound
// by the chain from the sequence to the page to its bounds. One row of 64 users with
// up to 1024 pages 12 us.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache_common.h"
#include "select_tiles.h"

namespace rs {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kPagesAtOnce = 64;  // of a wave
constexpr int kPageRun = kPagesAtOnce * (kBlock / kWave);

// A score's sign, exponent and first 20 bits: all of it.
__device__ inline uint32_t high_word(double x) { return static_cast<uint32_t>(__double2hiint(x)); }

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

// The q8 of LDS row `at`, by the 16 lanes of a quarter wave: `there` false leaves a
// row that no page's best comes from.
template <typename T, int W>
__device__ inline void quantise(const T* q, bool there, int d, int at, int part, char* q8, float* sq) {
  constexpr int E = W / 16, kStride = 2 * W + 16;  // E columns a lane; rows start on other banks
  float v[E];
  uint32_t top = 0;
  const bool in = there && part * E < d;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    v[i] = in ? to_f32(q[part * E + i]) : 0.0f;
    top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int i = 8; i > 0; i >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), i, kWave)));
  const bool bad = top >= 0x7F800000u;  // a query that is not finite finds every page alike
  const int k = bad ? 0 : unit_exp(__uint_as_float(top), 1.984375f, 6);
  const float inv = exp2_int(-k);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int w = bad ? 0 : static_cast<int>(rintf(v[i] * inv));
    q8[at * kStride + part * E + i] = static_cast<char>(max(w, 0));
    q8[at * kStride + W + part * E + i] = static_cast<char>(min(w, 0));
  }
  if (part == 0) sq[at] = there ? exp2_int(k) : -1.0f;
}

// Grid: runs of kPageRun pages, tiles of 1 << a.run_log rows of a sequence, key heads.
// LDS holds the q8 of kRowsAtOnce rows and heads, a row's heads to a multiple of 4 (of
// 16 past 8), so that a tile of the instruction is 4, 2 or 1 rows, or 16 heads of one.
constexpr int kRowsAtOnce = 64;
__host__ __device__ inline int heads_to(int group) { return group <= 4 ? 4 : group <= 8 ? 8 : (group + 15) & ~15; }  // LDS rows of a row
template <typename T, int W>
__global__ __launch_bounds__(kBlock) void k_select_score(const CacheSelect a) {
  constexpr int kSteps = 2 * W / 64, kGroups = kPagesAtOnce / 16, kStride = 2 * W + 16;
  extern __shared__ __align__(16) char score_lds[];
  float* sq = reinterpret_cast<float*>(score_lds);
  char* q8 = score_lds + kRowsAtOnce * sizeof(float);
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane & 15, grp = lane >> 4;
  const int kvh = blockIdx.z, run = 1 << a.run_log;
  int64_t tile;
  int s;
  if (c.pad > 0) {
    const uint32_t per = static_cast<uint32_t>(c.pad + run - 1) >> a.run_log, u = a.unit0 + blockIdx.y;
    s = static_cast<int>(u / per);
    tile = u - static_cast<uint32_t>(s) * per;
    if (s >= c.seqs) return;
  } else {
    s = find_tile(c.off, c.seqs, 1, a.run_log, a.unit0 + blockIdx.y, tile);
  }
  RowAt x;
  x.s = s;
  x.lk = cache_len(c, s);
  const SeqSpan span = seq_span(c.off, s, c.pad, c.rows);
  x.len = span.len;
  if (tile < 0 || tile * run >= span.len) return;  // block-uniform, as all below
  // the tile's rows in this launch
  const int64_t first_row = max(span.start + tile * run, a.row0);
  const int rows = static_cast<int>(min(min(span.start + min(tile * run + run, static_cast<int64_t>(span.len)), a.row0 + a.tokens) - first_row,
                                        static_cast<int64_t>(run)));
  if (rows <= 0) return;
  x.token = static_cast<int>(first_row - span.start) + rows - 1;
  const int most = pages_seen(a, x);  // of the last row, which sees the most
  if (most <= a.count) return;        // all of them
  const int slots = heads_to(a.group);
  const int held = min(slots, kRowsAtOnce);                                      // of them at once
  auto fill = [&](int h0) {
    for (int at = wave * 4 + grp; at < ((rows * held + 15) & ~15); at += 16) {
      const int own = at / held, head = h0 + at - own * held;
      const bool there = own < rows && head < a.group;
      const T* q = static_cast<const T*>(a.q.p) + (first_row + own) * a.q.row + static_cast<int64_t>(kvh * a.group + head) * a.q.head;
      quantise<T, W>(q, there, c.d, at, col, q8, sq);
    }
  };
  const bool once = slots <= kRowsAtOnce;
  bool filled = false;
  for (int page0 = blockIdx.x * kPageRun; page0 < most; page0 += gridDim.x * kPageRun) {
    const int first = page0 + wave * kPagesAtOnce;
    i32x4 box[kGroups][kSteps];
    float unit[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int n = first + i * 16 + col;
      const int page = n < most ? cache_page(c, s, n) : -1;
      const int64_t at = static_cast<int64_t>(max(page, 0)) * c.hkv + kvh;
      const int8_t* p = c.bounds + at * 2 * W + grp * 16;
      unit[i] = -INFINITY;  // a page that is not there comes last of all
#pragma unroll
      for (int k = 0; k < kSteps; ++k) box[i][k] = i32x4{0, 0, 0, 0};
      if (page >= 0) {
        unit[i] = c.units[at];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) box[i][k] = *reinterpret_cast<const i32x4*>(p + k * 64);
      }
    }
    if (once && !filled) {  // while the bounds are on their way
      fill(0);
      __syncthreads();
      filled = true;
    }
    // the best of a page over the 16 LDS rows from `base` on, for each group of four
    auto best_of = [&](int base, double (&best)[kGroups]) {
      i32x4 qa[kSteps];
      float scale[4];
#pragma unroll
      for (int k = 0; k < kSteps; ++k) qa[k] = *reinterpret_cast<const i32x4*>(q8 + (base + col) * kStride + k * 64 + grp * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) scale[e] = sq[base + grp * 4 + e];
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        i32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(qa[k], box[i][k], sum, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (scale[e] > 0.0f) best[i] = fmax(best[i], static_cast<double>(sum[e]) * static_cast<double>(scale[e]));
      }
    };
    auto write = [&](int own, bool mine, double (&best)[kGroups]) {
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        double y = best[i];
        if (slots >= 8) y = fmax(y, __shfl_xor(y, 16, kWave));
        if (slots >= 16) y = fmax(y, __shfl_xor(y, 32, kWave));
        const double score = unit[i] == -INFINITY ? -INFINITY : y * unit[i] + 0.0;  // one zero
        const int n = first + i * 16 + col;
        if (n < most && mine)
          a.scores[((first_row + own - a.row0) * c.hkv + kvh) * c.width + n] = high_word(score == score ? score : INFINITY);  // not finite: first
      }
    };
    if (slots <= 16) {
      for (int base = 0; base < rows * slots; base += 16) {
        double best[kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) best[i] = -INFINITY;
        best_of(base, best);
        const int own = (base + grp * 4) / slots;
        write(own, own < rows && (base + grp * 4) % slots == 0, best);
      }
    } else {
      for (int own = 0; own < rows; ++own) {
        double best[kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) best[i] = -INFINITY;
        for (int h0 = 0; h0 < slots; h0 += held) {
          if (!once) {  // more heads than LDS rows: one row at a time (run is 1)
            __syncthreads();
            fill(h0);
            __syncthreads();
          }
          for (int h = 0; h < held && h0 + h < slots; h += 16) best_of(own * held + h, best);
        }
        write(own, grp == 0, best);
      }
    }
  }
}

// Larger scores have larger keys.
__device__ inline uint32_t order(uint32_t b) { return b & 0x80000000u ? ~b : b | 0x80000000u; }

// A block per row and key head, its keys in registers: the count-th largest by
// halving the range of keys (a step is one compare a key and one barrier), then the
// pages above it and the first of those equal to it, in order. Bound by the latency of
// those steps: 64 of 15,625 pages 17 to 19 us (40 by histograms of the keys' bytes, which
// put most of like scores into a few counters; 25 with the range started at the least
// key), 32 of at most 1024 7.8.
template <int NT, int ITEMS>
__global__ __launch_bounds__(NT) void k_select_pick(const CacheSelect a) {
  constexpr int kWaves = NT / kWave;
  __shared__ int count_of[2][kWaves];
  __shared__ uint32_t top_of[kWaves], least_of[kWaves];
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
  const uint32_t* score = a.scores + (static_cast<int64_t>(blockIdx.x) * c.hkv + kvh) * c.width;
  uint32_t key[ITEMS];  // 0: no page (order gives no score 0)
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int n = i * NT + threadIdx.x;
    key[i] = n < seen ? order(score[n]) : 0;
    top = max(top, key[i]);
  }
  // The least of the largest keys of `count` groups of threads or more (none, if there are
  // fewer threads than that) has `count` keys from
  // it on, and a few times as many at most as a rule: most of the halving is done.
  uint32_t least = top;
#pragma unroll
  for (int i = 1; i < kWave; i <<= 1) {
    const uint32_t t = static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), i, kWave));
    const uint32_t l = static_cast<uint32_t>(__shfl_xor(static_cast<int>(least), i, kWave));
    top = max(top, t);
    least = a.count <= NT / (2 * i) ? max(least, l) : min(least, l);
  }
  if (lane == 0) {
    top_of[wave] = top;
    least_of[wave] = least;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    top = max(top, top_of[i]);
    least = min(least, least_of[i]);
  }
  // at least `count` keys are >= low, fewer are >= high; `above` of them
  uint32_t low = a.count <= NT ? max(least, 1u) : 1, high = top + 1;
  int above = 0, side = 0;
  while (high > low + 1) {
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
      if (n == a.count) {
        high = mid;
        above = n;
      }
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
      constexpr int kPer = (ITEMS * kWaves + kWave - 1) / kWave;
      int v[kPer], all = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        v[i] = lane * kPer + i < ITEMS * kWaves ? before[lane * kPer + i] : 0;
        all += v[i];
      }
      int run = wave_incl_scan(all) - all;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (lane * kPer + i < ITEMS * kWaves) before[lane * kPer + i] = run;
        run += v[i];
      }
    }
    __syncthreads();
  };
  static_assert(ITEMS <= 64, "a bit an item");
  uint64_t take = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) take |= uint64_t(key[i] >= high) << i;
  if (above < a.count) {  // scores that are equal
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint64_t equal = __ballot(key[i] >= low && key[i] < high);
      if (lane == 0) before[i * kWaves + wave] = static_cast<int>(__popcll(equal));
    }
    sums();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const bool equal = key[i] >= low && key[i] < high;
      const int rank = before[i * kWaves + wave] + static_cast<int>(__popcll(__ballot(equal) & below));
      take |= uint64_t(equal && rank < a.count - above) << i;
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint64_t taken = __ballot(take >> i & 1);
    if (lane == 0) before[i * kWaves + wave] = static_cast<int>(__popcll(taken));
  }
  sums();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const bool mine = take >> i & 1;
    const uint64_t taken = __ballot(mine);
    if (mine) out[before[i * kWaves + wave] + static_cast<int>(__popcll(taken & below))] = i * NT + threadIdx.x;
  }
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
  const uint32_t* score = a.scores + (static_cast<int64_t>(blockIdx.x) * c.hkv + kvh) * c.width;
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
constexpr int64_t kMostUnits = 65535;  // tiles lie along a launch's second axis

}  // namespace

size_t plan_cache_select(const CacheSelect& a, int64_t* tokens) {
  const size_t one = static_cast<size_t>(a.c.hkv) * std::max<int64_t>(a.c.width, 1) * sizeof(uint32_t);
  *tokens = 0;
  if (a.c.rows == 0 || a.c.seqs == 0) return 0;
  *tokens = std::min<int64_t>(a.c.rows, std::max<int64_t>(1, kMostScoreBytes / one));
  *tokens = std::min<int64_t>(*tokens, 65535);  // (a block each along the first axis of the picks)
  return *tokens * one;
}

template <typename T, int W>
static void run_select(const CacheSelect& a, hipStream_t s) {
  if (a.c.width > a.count) {
    const TileRange units = tiles_of_rows(a.c.seqs, a.c.rows, a.c.pad, a.run_log, a.row0, a.tokens);
    const int held = std::min(kRowsAtOnce, ((heads_to(a.group) << a.run_log) + 15) & ~15);
    const size_t lds = kRowsAtOnce * sizeof(float) + held * (2 * W + 16);
    CacheSelect b = a;
    for (int64_t u = 0; u < units.count; u += kMostUnits) {
      b.unit0 = static_cast<uint32_t>(units.first + u);
      const dim3 grid(a.tiles, static_cast<unsigned>(std::min(units.count - u, kMostUnits)), a.c.hkv);
      k_select_score<T, W><<<grid, kBlock, lds, s>>>(b);
    }
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
  a.run_log = tile_rows_log(a.c.seqs, a.c.rows, a.c.pad, tokens, kRowsAtOnce / heads_to(a.group));
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
