// Attention over ragged sequences, forward (gfx950).
//
//   s_ij = cap(scale q_i.k_j) - slope_h |p_i - j|, p_i = i + Lk - Lq
//   out_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp(s_ij)
//
// over the keys of the query's sequence that it sees.  One pass over the keys
// with the running maximum and sum of the softmax (Milakov & Gimelshein 2018),
// in base 2.  A block takes 128 packed rows (tokens times the query heads of
// one key head) and walks over the keys 64 at a time; a wave owns 32 rows, one
// per lane column: its maximum, sum and rescaling are the lane's own scalars.
// The next step's keys and values are requested before a step is computed; fp32
// runs beside them to the step's end, bf16 to its first transposed read of the
// values, before which the compiler waits for every load that writes LDS.  Where the rows alone make too few blocks (single tokens, short
// chunks), a block takes a chunk of the keys and a second kernel joins them.
//
// What bounds it.  Per score the products take 4 HD operations, which the matrix
// unit does in HD / 256 cycles a lane column, and the softmax 5 to 8 vector
// instructions (scale, maximum, exponent, sum, rounding; 3 more for a distance
// term, 8 for a cap, and two transcendental ones where a score passes its half): at HD = 128 the two are
// even, below it the vector unit bounds.  One causal sequence of 16384, 8 heads
// of 128 bf16: 561 to 594 us, 925 to 980 TFLOP/s of the scores it needs (a large
// library product reaches 1329); matrix unit 45% busy, vector unit 41%.  1536 padded
// sequences of 100 to 1024, 2 heads of 64, distances weighed: 426 us, vector unit
// 63% busy.  One token for each of 256 users, 8 heads of 128 over 2: 114 us, 4.5 TB/s with the join.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_common.h"

#pragma clang fp contract(fast)

namespace rs {
namespace {

// Blocks per CU that the registers are kept down for: one in its products while
// another is in its softmax (narrow rows fit three by themselves; held to four,
// they spill: 462 -> 724 us on the padded sequences); fp32 rows of 128 fill a CU.
template <typename T, int HD>
constexpr int kResidentBlocks = HD * sizeof(T) > 256 ? 1 : 2;

template <typename T, int HD, bool SPLIT>
__global__ __launch_bounds__(kAttnWaves* kWave, (kResidentBlocks<T, HD>)) void k_attn_fwd(const AttnArgs a) {
  typedef Tile<T, HD> L;
  typedef typename Frag<T>::type F;
  constexpr int KS = HD / 16;  // product steps over d
  constexpr int DT = HD / 32;  // 32-column tiles of the output
  constexpr int kTile = kAttnStep * L::kRowBytes;
  __shared__ __align__(1024) char lds[4 * kTile];  // keys and values, two steps of each

  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int half = lane >> 5, col = lane & 31;
  int kvh = blockIdx.y;
  int s;
  int64_t tile;
  int c0 = 0;  // the block's first key
  BlockOf blk{};
  if (!SPLIT) {
    blk = block_of(a, true);
    kvh = blk.kvh;
  }
  if (SPLIT) {
    int64_t c;
    if (a.kv_pad > 0) {
      const uint32_t per = static_cast<uint32_t>(a.kv_pad + a.chunk - 1) / a.chunk;
      s = blockIdx.x / per;
      c = blockIdx.x - s * per;
    } else {
      s = find_seq(a.kv_off, a.seqs, 1, a.chunk, blockIdx.x, c);
    }
    tile = blockIdx.z;
    if (c < 0 || c * a.chunk >= int64_t(1) << 31) return;
    c0 = static_cast<int>(c) * a.chunk;
  } else if (a.q_pad > 0) {
    const uint32_t per = static_cast<uint32_t>((a.q_pad * a.group + kAttnRows - 1) / kAttnRows);
    s = static_cast<uint32_t>(blk.tile) / per;
    tile = blk.tile - static_cast<int64_t>(s) * per;
  } else {
    s = find_seq(a.q_off, a.seqs, a.group, kAttnRows, blk.tile, tile);
  }
  const SeqSpan qs = seq_span(a.q_off, s, a.q_pad, a.q_rows), ks = seq_span(a.kv_off, s, a.kv_pad, a.kv_rows);
  const int rows = qs.len * a.group;  // the others of a padded sequence have no key
  const int64_t out_rows = a.q_pad > 0 ? a.q_pad * a.group : rows;
  if (tile < 0 || tile * kAttnRows >= out_rows) return;  // block-uniform
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;

  const int r0 = static_cast<int>(tile) * kAttnRows;
  const int r = r0 + wave * 32 + col;  // the lane's row
  const RowOf me = row_of(r, kvh, a.group);
  const bool live = r < rows;
  const int limit = live ? key_limit(me.token, qs.len, ks.len, a.causal, prefix) : 0;
  // limits do not fall along the rows: the last row sees the most keys
  const int last = min(r0 + kAttnRows, rows) - 1;
  int end = last >= r0 ? key_limit(div_group(last, a.group), qs.len, ks.len, a.causal, prefix) : 0;
  const bool joined = SPLIT && ks.len > a.chunk;  // other blocks hold parts of these rows
  if (SPLIT) {
    if (c0 > 0 && c0 >= end) return;  // block-uniform; the join does not look here
    end = c0 + min(end - c0, a.chunk);  // c0 + chunk may pass 2^31
  }
  const int w0 = r0 + wave * 32, w1 = min(w0 + 32, rows) - 1;
  const int wave_least = w0 < rows ? key_limit(div_group(w0, a.group), qs.len, ks.len, a.causal, prefix) : 0;
  const int wave_most = w1 >= w0 ? key_limit(div_group(w1, a.group), qs.len, ks.len, a.causal, prefix) : 0;

  TileLoader<T, HD> kl, vl;
  kl.init(a.k.p, ks.start, a.k.row, kvh * a.k.head, a.d, ks.len);
  vl.init(a.v.p, ks.start, a.v.row, kvh * a.v.head, a.d, ks.len);
  if (c0 < end) {
    kl.load(lds, c0);
    vl.load(lds + 2 * kTile, c0);
  }
  F qf[KS];
  {
    const T* q = static_cast<const T*>(a.q.p) + (qs.start + me.token) * a.q.row + me.head * a.q.head;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int k0 = t * 16 + half * 8;
      qf[t] = zero_frag<T>();
      if (live && k0 < a.d) load_frag(q + k0, qf[t]);
    }
  }
  const int pos = me.token + ks.len - qs.len;
  const int wave_pos0 = div_group(w0, a.group) + ks.len - qs.len;
  const int wave_pos1 = div_group(max(w1, w0), a.group) + ks.len - qs.len;
  const float slope = a.slopes && live ? a.slopes[me.head] * kLog2e : 0.0f;
  const float inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap2 = a.cap * kLog2e, scale2 = a.scale * kLog2e;
  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x16{};
  // the running maximum in base 2 and the height above it at which it moves:
  // any, while no key has been seen
  float m = 0.0f, move = -INFINITY, l = 0.0f;

  int buf = 0;
  for (int j0 = c0; j0 < end; j0 += kAttnStep, buf ^= 1) {
    wait_tiles();  // this step's tiles are there, the other step's have been read
    if (j0 + kAttnStep < end) {
      kl.load(lds + (buf ^ 1) * kTile, j0 + kAttnStep);
      vl.load(lds + (2 + (buf ^ 1)) * kTile, j0 + kAttnStep);
    }
    if (j0 >= wave_most) continue;  // wave-uniform: none of its rows sees these keys
    const char* kt = lds + buf * kTile;
    const char* vt = lds + (2 + buf) * kTile;

    float p[2][16];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 sc = {};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        F kf;
        row_frag<HD>(kt, kb * 32 + col, t * 16 + half * 8, kf);
        sc = mma(kf, qf[t], sc);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) p[kb][i] = sc[i];
    }
    // in base 2, relative to the running maximum
    const int j = j0 + half * 4;  // register i of block kb is key j + kb * 32 + (i / 4) * 8 + i % 4
    float c = scale2;
    if (a.cap > 0.0f) {
      c = cap2;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) tanh_scores<T>(p[kb], inv_cap);
    }
    if (!a.slopes) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) p[kb][i] = p[kb][i] * c - m;
    } else {
      const float dist = static_cast<float>(j - pos);
      const int sign = dist_sign(j0, j0 + kAttnStep - 1, wave_pos0, wave_pos1);
      if (sign != 0) {
        const float e = sign > 0 ? slope : -slope, b = dist * e - m;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            p[kb][i] = p[kb][i] * c + (e * static_cast<float>(kb * 32 + (i >> 2) * 8 + (i & 3)) + b);
      } else {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            p[kb][i] = p[kb][i] * c - (slope * fabsf(dist + static_cast<float>(kb * 32 + (i >> 2) * 8 + (i & 3))) + m);
      }
    }
    if (j0 + kAttnStep > wave_least) {
      const int left = limit - j;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          p[kb][i] = kb * 32 + (i >> 2) * 8 + (i & 3) < left ? p[kb][i] : -INFINITY;
    }
    float top = p[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, p[kb][i]);
    top = other_half_max(top);
    // the running maximum moves only when a score passes it by 2^8: until then
    // the probabilities are larger than 1 by at most that, which neither fp32
    // sums nor bf16's relative rounding notice
    if (__any(top > move)) {
      const bool up = top > move;
      const float by = up ? top : 0.0f;
      const float alpha = move == -INFINITY ? 0.0f : exp2_hw(-by);
      m += by;
      move = up ? 8.0f : move;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i) acc[i] *= alpha;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) p[kb][i] -= by;
    }
    float sum = 0.0f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[kb][i] = exp2_hw(p[kb][i]);
        sum += p[kb][i];
      }
    l += sum;  // this half's keys
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const F pf = to_frag<T>(p[kb], t);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          F vf;
          col_frag<HD>(vt, kb * 32 + t * 16, i * 32, lane, vf);
          acc[i] = mma(vf, pf, acc[i]);
        }
      }
  }

  l = other_half_sum(l);
  if (joined) {
    const int at = wave * 32 + col;
    if (r >= out_rows || at >= a.part_rows) return;
    const int64_t slot = ((static_cast<int64_t>(blockIdx.x) * a.hkv + kvh) * a.row_tiles + tile) * a.part_rows + at;
    float* po = a.part_o + slot * a.d;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d0 = i * 32 + g * 8 + half * 4;
        if (d0 < a.d) store4(po + d0, acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]);
      }
    if (half == 0) reinterpret_cast<float2*>(a.part_ml)[slot] = make_float2(m, l);
    return;
  }
  const bool none = !live || l == 0.0f;  // no key: 0 (a NaN sum stays)
  const float inv = none ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = none ? 0.0f : acc[i][e] * inv;
  typedef RowWriter<T, HD> S;
  static_assert(S::kBytes <= kTile, "a wave's rows fit its share of the tiles");
  __syncthreads();  // the tiles have been read
  char* mine = lds + wave * kTile;
  S::put(mine, lane, [&](int i, int e) { return acc[i][e]; });
  auto at = [&](void* base, int64_t end_row, int i) -> T* {
    if (w0 + i >= end_row) return nullptr;
    const RowOf x = row_of(w0 + i, kvh, a.group);
    return static_cast<T*>(base) + ((qs.start + x.token) * a.hq + x.head) * a.d;
  };
  S::flush(mine, lane, a.d, [&](int i) { return at(a.out, out_rows, i); });
  if (sizeof(T) == 2 && a.rest) {
    S::put(mine, lane, [&](int i, int e) { return rest_bf16(acc[i][e]); });
    S::flush(mine, lane, a.d, [&](int i) { return at(a.rest, rows, i); });
  }
  if (a.lse && half == 0 && r < out_rows)
    a.lse[(qs.start + me.token) * a.hq + me.head] = none ? -INFINITY : m * kLn2 + logf(l);
}

// At most 32 rows a sequence and key head (single tokens, a few candidates):
// bound by reading the keys and values once.  A wave walks over blocks of 32
// keys of its own, W waves in turn through the block's chunk, with its own
// place for a block's keys and one for its values in LDS: the next keys are on
// their way as soon as the scores are taken, the next values as soon as the
// output is, and no barrier ties the waves together.  The waves' results are
// joined as those of chunks are.  Four candidates over 1,000,003 keys, two key
// heads of 64 bf16: 90 us, 5.7 TB/s (reads alone reach 6.8).
template <typename T, int HD>
struct FewShape {
  static constexpr int W = 8;
  static constexpr bool kUsed = HD * sizeof(T) <= 128;
};

template <typename T, int HD>
__global__ __launch_bounds__((FewShape<T, HD>::W * kWave)) void k_attn_few(const AttnArgs a) {
  typedef FewShape<T, HD> C;
  typedef Tile<T, HD> L;
  typedef typename Frag<T>::type F;
  constexpr int KS = HD / 16, DT = HD / 32;
  constexpr int kTile = 32 * L::kRowBytes;
  __shared__ __align__(1024) char k_place[C::W * kTile], v_place[C::W * kTile];
  __shared__ float2 sh_ml[C::W][32];

  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int half = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.y;
  int s;
  int64_t ci;
  if (a.kv_pad > 0) {
    const uint32_t per = static_cast<uint32_t>(a.kv_pad + a.chunk - 1) / a.chunk;
    s = blockIdx.x / per;
    ci = blockIdx.x - s * per;
  } else {
    s = find_seq(a.kv_off, a.seqs, 1, a.chunk, blockIdx.x, ci);
  }
  if (ci < 0 || ci * a.chunk >= int64_t(1) << 31) return;
  const int c0 = static_cast<int>(ci) * a.chunk;
  const SeqSpan qs = seq_span(a.q_off, s, a.q_pad, a.q_rows), ks = seq_span(a.kv_off, s, a.kv_pad, a.kv_rows);
  const int rows = min(qs.len * a.group, a.part_rows);
  const int out_rows = a.q_pad > 0 ? a.part_rows : rows;
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;
  const RowOf me = row_of(col, kvh, a.group);
  const bool live = col < rows;
  const int limit = live ? key_limit(me.token, qs.len, ks.len, a.causal, prefix) : 0;
  int end = rows > 0 ? key_limit(div_group(rows - 1, a.group), qs.len, ks.len, a.causal, prefix) : 0;
  const int least = rows > 0 ? key_limit(0, qs.len, ks.len, a.causal, prefix) : 0;
  const bool joined = ks.len > a.chunk;
  if (c0 > 0 && c0 >= end) return;  // block-uniform; the join does not look here
  end = c0 + min(end - c0, a.chunk);  // c0 + chunk may pass 2^31

  // the wave's blocks of 32 keys: first, first + 32 W, ...
  const int first = c0 + wave * 32;
  const int n_mine = first < end ? (end - first + 32 * C::W - 1) / (32 * C::W) : 0;
  char *kt = k_place + wave * kTile, *vt = v_place + wave * kTile;
  TileLoader<T, HD, 32, 1> kl, vl;
  kl.init(a.k.p, ks.start, a.k.row, kvh * a.k.head, a.d, ks.len);
  vl.init(a.v.p, ks.start, a.v.row, kvh * a.v.head, a.d, ks.len);
  constexpr int kLoads = TileLoader<T, HD, 32, 1>::kLoads;  // of a block of keys, or of values
  if (n_mine > 0) {
    kl.load(kt, first);
    vl.load(vt, first);
  }
  F qf[KS];
  {
    const T* q = static_cast<const T*>(a.q.p) + (qs.start + me.token) * a.q.row + me.head * a.q.head;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int k0 = t * 16 + half * 8;
      qf[t] = zero_frag<T>();
      if (live && k0 < a.d) load_frag(q + k0, qf[t]);
    }
  }
  const int pos = me.token + ks.len - qs.len;
  const float slope = a.slopes && live ? a.slopes[me.head] * kLog2e : 0.0f;
  const float inv_cap = a.cap > 0.0f ? a.scale / a.cap : 0.0f, cap2 = a.cap * kLog2e, scale2 = a.scale * kLog2e;

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x16{};
  float m = 0.0f, move = -INFINITY, l = 0.0f;

  for (int n = 0; n < n_mine; ++n) {
    const int j0 = first + n * 32 * C::W;
    const bool more = n + 1 < n_mine;
    wait_loads<kLoads>();  // the keys have arrived, the values may be on their way
    asm volatile("" ::: "memory");
    f32x16 sc = {};
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      F kf;
      row_frag<HD>(kt, col, t * 16 + half * 8, kf);
      sc = mma(kf, qf[t], sc);
    }
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = sc[i];
    if (more) kl.load(kt, j0 + 32 * C::W);  // the products have read the keys
    const int j = j0 + half * 4;  // register i is key j + (i / 4) * 8 + i % 4
    float c = scale2;
    if (a.cap > 0.0f) {
      c = cap2;
      tanh_scores<T>(p, inv_cap);
    }
    if (!a.slopes) {
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = p[i] * c - m;
    } else {
      const float dist = static_cast<float>(j - pos);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        p[i] = p[i] * c - (slope * fabsf(dist + static_cast<float>((i >> 2) * 8 + (i & 3))) + m);
    }
    if (j0 + 32 > least || j0 + 32 > end) {
      const int left = min(limit, end) - j;
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = (i >> 2) * 8 + (i & 3) < left ? p[i] : -INFINITY;
    }
    float top = p[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, p[i]);
    top = other_half_max(top);
    if (__any(top > move)) {
      const bool up = top > move;
      const float by = up ? top : 0.0f;
      const float alpha = move == -INFINITY ? 0.0f : exp2_hw(-by);
      m += by;
      move = up ? 8.0f : move;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i) acc[i] *= alpha;
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] -= by;
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = exp2_hw(p[i]);
      sum += p[i];
    }
    l += sum;
    if (more) wait_loads<kLoads>();  // the values
    else wait_loads<0>();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const F pf = to_frag<T>(p, t);
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        F vf;
        col_frag<HD>(vt, t * 16, i * 32, lane, vf);
        acc[i] = mma(vf, pf, acc[i]);
      }
    }
    if (more) vl.load(vt, j0 + 32 * C::W);  // the products have read the values
  }

  // the waves' parts: m = max m_w, acc = sum acc_w 2^(m_w - m), l alike
  l = other_half_sum(l);
  if (half == 0) sh_ml[wave][col] = make_float2(m, l);
  __syncthreads();  // and the rings have been read
  float m_all = -INFINITY;
#pragma unroll
  for (int w = 0; w < C::W; ++w) m_all = fmaxf(m_all, sh_ml[w][col].y == 0.0f ? -INFINITY : sh_ml[w][col].x);
  const float base = m_all == -INFINITY ? 0.0f : m_all;
  const float mul = l == 0.0f ? 0.0f : exp2_hw(m - base);
  constexpr int kPart = DT * 16 * kWave * sizeof(float);
  static_assert(C::W / 2 * kPart <= static_cast<int>(sizeof(k_place)), "half of the parts fit");
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] *= mul;
#pragma unroll
  for (int w = C::W / 2; w >= 1; w /= 2) {  // the upper half of the waves hand theirs to the lower half
    f32x4* at = reinterpret_cast<f32x4*>(k_place + wave % w * kPart) + lane;
    if (wave >= w && wave < 2 * w)
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          at[(i * 4 + e) * kWave] = f32x4{acc[i][4 * e], acc[i][4 * e + 1], acc[i][4 * e + 2], acc[i][4 * e + 3]};
    __syncthreads();
    if (wave < w)
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4 x = at[(i * 4 + e) * kWave];
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[i][4 * e + q] += x[q];
        }
    __syncthreads();
  }
  if (wave > 0) return;
  l = 0.0f;
#pragma unroll
  for (int w = 0; w < C::W; ++w) {
    const float2 x = sh_ml[w][col];
    l += x.y == 0.0f ? 0.0f : x.y * exp2_hw(x.x - base);
  }
  m = base;
  if (col >= out_rows) return;
  if (joined) {
    const int64_t slot = (static_cast<int64_t>(blockIdx.x) * a.hkv + kvh) * a.part_rows + col;
    float* po = a.part_o + slot * a.d;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d0 = i * 32 + g * 8 + half * 4;
        if (d0 < a.d) store4(po + d0, acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]);
      }
    if (half == 0) reinterpret_cast<float2*>(a.part_ml)[slot] = make_float2(m, l);
    return;
  }
  const bool none = !live || l == 0.0f;
  const float inv = none ? 0.0f : 1.0f / l;
  const int64_t row = (qs.start + me.token) * a.hq + me.head;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d0 = i * 32 + g * 8 + half * 4;
      if (d0 >= a.d) continue;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = none ? 0.0f : acc[i][4 * g + e] * inv;
      store4(static_cast<T*>(a.out) + row * a.d + d0, x[0], x[1], x[2], x[3]);
      if (sizeof(T) == 2 && a.rest && live)
        store4(static_cast<T*>(a.rest) + row * a.d + d0, rest_bf16(x[0]), rest_bf16(x[1]), rest_bf16(x[2]), rest_bf16(x[3]));
    }
  if (a.lse && half == 0) a.lse[row] = none ? -INFINITY : m * kLn2 + logf(l);
}

// Two consecutive elements, as floats and from them.
__device__ inline float2 load2(const float* p) { return *reinterpret_cast<const float2*>(p); }
__device__ inline float2 load2(const uint16_t* p) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ inline void store2(float* p, float a, float b) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }
__device__ inline void store2(uint16_t* p, float a, float b) { *reinterpret_cast<uint32_t*>(p) = pack_bf16(a, b); }

// A row of the split that no part holds, since its sequence has more queries than
// the caller's bound: a block takes it over all its keys, a wave a key at a time,
// a lane two columns.  Slow, but such rows are a caller's mistake.
template <typename T, int NT>
__device__ __forceinline__ void whole_row(const AttnArgs& a, const SeqSpan& qs, const SeqSpan& ks, int token, int head, int kvh,
                                 int limit, float2* sh_o, float2* sh_ml) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, c = 2 * lane;
  const bool in = c < a.d;
  const T* q = static_cast<const T*>(a.q.p) + (qs.start + token) * a.q.row + head * a.q.head + c;
  const float2 none = make_float2(0.0f, 0.0f), qv = in ? load2(q) : none;
  const int pos = token + ks.len - qs.len;
  const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
  float m = -INFINITY, l = 0.0f;
  float2 o = none;
  for (int j = wave; j < limit; j += NT / kWave) {
    const T* k = static_cast<const T*>(a.k.p) + (ks.start + j) * a.k.row + kvh * a.k.head + c;
    const T* v = static_cast<const T*>(a.v.p) + (ks.start + j) * a.v.row + kvh * a.v.head + c;
    const float2 kv = in ? load2(k) : none, vv = in ? load2(v) : none;
    float x = qv.x * kv.x + qv.y * kv.y;
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) x += __shfl_xor(x, d, kWave);
    x = a.cap > 0.0f ? a.cap * kLog2e * tanhf(x * (a.scale / a.cap)) : x * (a.scale * kLog2e);
    x -= slope * fabsf(static_cast<float>(j - pos));
    const float top = fmaxf(m, x), base = top == -INFINITY ? 0.0f : top;
    const float alpha = exp2_hw(m - base), p = exp2_hw(x - base);
    m = top;
    l = l * alpha + p;
    o.x = o.x * alpha + p * vv.x;
    o.y = o.y * alpha + p * vv.y;
  }
  sh_o[threadIdx.x] = o;
  if (lane == 0) sh_ml[wave] = make_float2(m, l);
  __syncthreads();
  if (wave > 0) return;
  m = -INFINITY;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) m = fmaxf(m, sh_ml[w].x);
  l = 0.0f;
  o = none;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) {
    const float mul = sh_ml[w].y == 0.0f ? 0.0f : exp2_hw(sh_ml[w].x - m);
    const float2 x = sh_o[w * kWave + lane];
    l += mul * sh_ml[w].y;
    o.x += mul * x.x;
    o.y += mul * x.y;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int64_t row = (qs.start + token) * a.hq + head;
  if (in) {
    store2(static_cast<T*>(a.out) + row * a.d + c, o.x * inv, o.y * inv);
    if (sizeof(T) == 2 && a.rest)
      store2(static_cast<T*>(a.rest) + row * a.d + c, rest_bf16(o.x * inv), rest_bf16(o.y * inv));
  }
  if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
}

// Joins the chunks of a row: a block per query token and head, threads four
// columns and a share of the chunks each.  Bound by the latency of its two trips
// (maxima, then parts): 9 us for 2048 rows of few chunks, 10 for 16 rows of 245.
//   m = max m_c,  l = sum l_c 2^(m_c - m),  out = sum acc_c 2^(m_c - m) / l
template <typename T, int NT>
__global__ __launch_bounds__(NT) void k_attn_join(const AttnArgs a) {
  __shared__ float4 sh_o[NT];
  __shared__ __align__(8) float sh_l[NT];
  __shared__ float sh_m[NT / kWave];
  const int head = blockIdx.y, kvh = head / a.group;
  int s;
  int64_t token;
  if (a.q_pad > 0) {
    s = static_cast<int>(blockIdx.x / a.q_pad);
    token = blockIdx.x - s * a.q_pad;
  } else {
    s = find_seq(a.q_off, a.seqs, 1, 1, blockIdx.x, token);
  }
  const SeqSpan qs = seq_span(a.q_off, s, a.q_pad, a.q_rows), ks = seq_span(a.kv_off, s, a.kv_pad, a.kv_rows);
  if (token < 0 || token >= (a.q_pad > 0 ? a.q_pad : int64_t(qs.len))) return;  // no row; block-uniform, as below
  const int r = static_cast<int>(token) * a.group + head - kvh * a.group;
  const int64_t tile = r / kAttnRows, at = r % kAttnRows;
  const bool past = tile >= a.row_tiles || at >= a.part_rows;  // of the caller's bound of the queries
  if (!past && ks.len <= a.chunk) return;                      // written
  const int prefix = a.prefix ? static_cast<int>(min(max(a.prefix[s], int64_t(0)), int64_t(ks.len))) : 0;
  const int limit = token < qs.len ? key_limit(static_cast<int>(token), qs.len, ks.len, a.causal, prefix) : 0;
  if (__builtin_expect(past, 0)) {
    // the arguments again, by an address that is not known before: the compiler else
    // loads q, k and v ahead of the branch, and every row waits for a further line of
    // the arguments (9.0 -> 10.0 us)
    uint64_t args = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());
    asm volatile("" : "+s"(args));
    whole_row<T, NT>(*reinterpret_cast<const AttnArgs*>(args), qs, ks, static_cast<int>(token), head, kvh, limit, reinterpret_cast<float2*>(sh_o),
                     reinterpret_cast<float2*>(sh_l));
    return;
  }
  const int chunks = static_cast<int>((static_cast<uint32_t>(limit) + a.chunk - 1) / a.chunk);
  const int64_t first = a.kv_pad > 0 ? s * ((a.kv_pad + a.chunk - 1) / a.chunk) : tile_base(a.kv_off, s, 1, a.chunk);
  const int64_t slot0 = ((first * a.hkv + kvh) * a.row_tiles + tile) * a.part_rows + at;
  const int64_t step = static_cast<int64_t>(a.hkv) * a.row_tiles * a.part_rows;

  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  float m = -INFINITY;
  for (int c = threadIdx.x; c < chunks; c += NT) {
    const float2 x = ml[slot0 + c * step];
    m = fmaxf(m, x.y == 0.0f ? -INFINITY : x.x);  // a part may see no key
  }
#pragma unroll
  for (int d = kWave / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
  if ((threadIdx.x & (kWave - 1)) == 0) sh_m[threadIdx.x / kWave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) m = fmaxf(m, sh_m[w]);
  const float base = m == -INFINITY ? 0.0f : m;

  const int quads = a.d / 4;  // at most 32
  const int shares = NT / quads, q = threadIdx.x % quads, share = threadIdx.x / quads;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float l = 0.0f;
  if (share < shares) {
#pragma unroll 4
    for (int c = share; c < chunks; c += shares) {
      const int64_t slot = slot0 + c * step;
      const float2 x = ml[slot];
      const float4 y = *reinterpret_cast<const float4*>(a.part_o + slot * a.d + 4 * q);
      const float w = x.y == 0.0f ? 0.0f : exp2_hw(x.x - base);
      l += w * x.y;
      o.x += w * y.x;
      o.y += w * y.y;
      o.z += w * y.z;
      o.w += w * y.w;
    }
  }
  sh_o[threadIdx.x] = o;
  sh_l[threadIdx.x] = l;
  __syncthreads();
  if (share > 0) return;
  for (int k = 1; k < shares; ++k) {
    const float4 y = sh_o[k * quads + q];
    l += sh_l[k * quads + q];
    o.x += y.x;
    o.y += y.y;
    o.z += y.z;
    o.w += y.w;
  }
  const bool none = l == 0.0f;
  const float inv = none ? 0.0f : 1.0f / l;
  const int64_t row = (qs.start + token) * a.hq + head;
  const float x[4] = {none ? 0.0f : o.x * inv, none ? 0.0f : o.y * inv, none ? 0.0f : o.z * inv, none ? 0.0f : o.w * inv};
  store4(static_cast<T*>(a.out) + row * a.d + 4 * q, x[0], x[1], x[2], x[3]);
  if (sizeof(T) == 2 && a.rest)
    store4(static_cast<T*>(a.rest) + row * a.d + 4 * q, rest_bf16(x[0]), rest_bf16(x[1]), rest_bf16(x[2]), rest_bf16(x[3]));
  if (a.lse && q == 0) a.lse[row] = none ? -INFINITY : m * kLn2 + logf(l);
}

int64_t key_chunks(const AttnArgs& a) {
  if (a.kv_pad > 0) return a.seqs * ((a.kv_pad + a.chunk - 1) / a.chunk);
  return a.kv_rows / a.chunk + a.seqs;
}

template <typename T, int HD>
hipError_t run(const AttnArgs& a, hipStream_t s) {
  if (a.chunk > 0) {
    const dim3 grid(static_cast<unsigned>(key_chunks(a)), a.hkv, a.row_tiles);
    if constexpr (FewShape<T, HD>::kUsed) {
      if (a.few) k_attn_few<T, HD><<<grid, FewShape<T, HD>::W * kWave, 0, s>>>(a);
      else k_attn_fwd<T, HD, true><<<grid, kAttnWaves * kWave, 0, s>>>(a);
    } else {
      k_attn_fwd<T, HD, true><<<grid, kAttnWaves * kWave, 0, s>>>(a);
    }
    const dim3 jg(static_cast<unsigned>(a.q_pad > 0 ? a.q_rows : a.q_rows + a.seqs), a.hq);
    // threads by the chunks of a row: many rows of few chunks, or few rows of many
    if (key_chunks(a) / a.seqs > 32) k_attn_join<T, 1024><<<jg, 1024, 0, s>>>(a);
    else k_attn_join<T, 128><<<jg, 128, 0, s>>>(a);
  } else {
    launch_blocks<kAttnWaves * kWave>(k_attn_fwd<T, HD, false>, a, attn_row_tiles(a) * a.hkv, s);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t run_type(const AttnArgs& a, hipStream_t s) {
  if (a.d <= 32) return run<T, 32>(a, s);
  if (a.d <= 64) return run<T, 64>(a, s);
  return run<T, 128>(a, s);
}

}  // namespace

int64_t attn_row_tiles(const AttnArgs& a) {
  if (a.seqs == 0) return 0;
  if (a.q_pad > 0) return a.seqs * ((a.q_pad * a.group + kAttnRows - 1) / kAttnRows);
  return a.q_rows * a.group / kAttnRows + a.seqs;
}

// Split where the row tiles alone leave CUs without a block: fewer than
// kFewBlocks, or for at most 32 rows a sequence and key head, whose parts are
// small next to the keys, kFewRowBlocks.  (Kernel and join against one pass, 128
// bf16: 88 row tiles, chunks of 33 to 257 queries over 2000 to 8191 keys, 59 + 19
// and 174 us; 376 tiles, 200 to 300 queries over 2000 to 4000, 58 + 44 and 78; 512
// tiles, four sequences of 4000, 104 + 80 and 127.)
// About kSplitBlocks blocks (kFewSplitBlocks of k_attn_few's larger ones) of at
// least kLeastChunk keys: more read no faster and leave more parts to join (that
// chunk case 61 + 22 with 2048, 59 + 19 with 1024, 60 + 18 with 512; one token
// of 256 users 115 + 9, 116 + 9, 130 + 8; a million keys (k_attn_few) 111 + 20 with
// 2048, 97 + 14 with 1024, 94 + 10 with 512).
constexpr int64_t kFewBlocks = 256, kFewRowBlocks = 1024;
constexpr int64_t kSplitBlocks = 1024, kFewSplitBlocks = 512, kLeastChunk = 256;
// Where no bound of the queries is known the parts' room follows the largest
// sequence that the rows allow; past this it is not taken.
constexpr size_t kMostPartBytes = size_t(256) << 20;
// Short sequences on the average are not split (nothing to join: 64 sessions of
// up to 50 keys 7.6 + 3.5 -> 7.6 us) unless the keys are many enough for a long
// one among them to matter.
constexpr int64_t kShortKeyRows = 8192;

// Whether k_attn_few takes the split: at most 32 rows, of at most 128 bytes.  (One
// candidate set over a million keys of 64 bf16: 115 us in 64-key steps of the
// general kernel, 95 so; one token of 256 users, 128 bf16, 113 and 120.)
static bool attn_few_rows(const AttnArgs& a, int64_t most_q) {
  const int width = a.d <= 32 ? 32 : a.d <= 64 ? 64 : 128;
  return most_q * a.group <= 32 && width * (a.bf16 ? 2 : 4) <= 128;
}

size_t plan_attn_split(AttnArgs* a, int64_t max_q, size_t* ml_at) {
  a->chunk = 0;
  *ml_at = 0;
  if (a->seqs == 0 || a->q_rows == 0) return 0;
  int64_t most_q = a->q_pad > 0 ? a->q_pad : a->q_rows;
  if (a->q_pad == 0 && max_q > 0) most_q = std::min(most_q, max_q);
  if (attn_row_tiles(*a) * a->hkv >= (most_q * a->group <= 32 ? kFewRowBlocks : kFewBlocks)) return 0;
  const int64_t most_keys = a->kv_pad > 0 ? a->kv_pad : a->kv_rows;  // of one sequence
  if (most_keys < 2 * kLeastChunk || (a->kv_rows < kShortKeyRows && a->kv_rows / a->seqs < kLeastChunk)) return 0;
  const int64_t tiles = (most_q * a->group + kAttnRows - 1) / kAttnRows;
  const int64_t share = a->kv_rows * a->hkv * tiles / (attn_few_rows(*a, most_q) ? kFewSplitBlocks : kSplitBlocks);
  const int64_t chunk = std::max(kLeastChunk, (share + kAttnStep - 1) / kAttnStep * kAttnStep);
  if (chunk >= most_keys) return 0;
  a->chunk = static_cast<int>(chunk);
  a->row_tiles = static_cast<int>(tiles);
  a->few = attn_few_rows(*a, most_q);
  a->part_rows = static_cast<int>(std::min(most_q * a->group, int64_t(kAttnRows)));
  const size_t slots = static_cast<size_t>(key_chunks(*a)) * a->hkv * a->row_tiles * a->part_rows;
  *ml_at = (slots * a->d * sizeof(float) + 255) / 256 * 256;
  const size_t bytes = *ml_at + slots * 2 * sizeof(float);
  if (bytes <= kMostPartBytes) return bytes;
  a->chunk = 0;
  return 0;
}

hipError_t launch_attn_fwd(const AttnArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? run_type<uint16_t>(a, s) : run_type<float>(a, s);
}

}  // namespace rs
