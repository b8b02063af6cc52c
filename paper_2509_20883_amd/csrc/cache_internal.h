// Declarations shared by the kernels of the paged sequence cache and their C
// ABI entry points.
//
// A page holds page_len tokens (32 to 256, a power of two) of every key head,
// its keys and its values, in 8 bits, in the order in which a wave's 16-byte
// loads hand them to the matrix instructions (W: the head's columns, padded to
// 32, 64 or 128 with zeros):
//   keys    [W / 16][page_len][16]   16 columns of one token together
//   values  [page_len / 16][W][16]   16 tokens of one column together
// so a product over columns (scores) and one over tokens (the output) both find
// their long side in a lane's own bytes.
#pragma once

#include "seq_internal.h"

namespace rs {

constexpr int kCacheBlock = 32;  // tokens a wave takes at a time

// The cache and the sequences of a call, as the kernels see them.
struct CacheArgs {
  uint8_t* data;   // [pages][hkv][2][page_len * W]
  float* scales;   // [pages][hkv][2], both 0: tokens lost, a page that is passed over
  void* open;      // [slots][2][hkv][2][page_len][d]
  int8_t* bounds;  // [pages][hkv][2][W] column maxima, minima; or null
  float* units;    // [pages][hkv], -inf where tokens are lost
  int64_t pages, slots;
  int hkv, d, plog;  // page_len = 1 << plog
  const int64_t *off, *lens;
  const int32_t *table, *slot_of;
  int64_t width, rows, pad;
  int seqs;
};

struct CacheAppend {
  CacheArgs c;
  HeadRows k, v, q;  // k.p null: no tokens are written; q.p null: none to turn
  int hq, rotary, next;
  const uint64_t* turns;
  void* q_out;
  int64_t* new_lens;
  int64_t page_units, q_units;  // blocks of the grid's two first parts
  int64_t block0;
};

struct CacheRead {
  CacheArgs c;  // off, rows: of the rows read
  const int64_t* start;
  void *k, *v;
  bool out_bf16;
};

struct CacheAttn {
  CacheArgs c;
  HeadRows q;
  int hq, group, causal;
  float scale, cap;
  const float* slopes;
  const int32_t* list;  // [rows][hkv][count] page numbers of a sequence, or null
  int count;
  void* out;
  int tile_log;  // rows of a block, 1 << tile_log: 16 or 32, its waves along the keys, or 128, along the rows
  int splits;    // blocks that share a row tile's keys
  int64_t units;
  uint32_t unit0;
  float *part_o, *part_ml;
};

struct CacheSelect {
  CacheArgs c;
  HeadRows q;
  int hq, group, causal, count;
  int32_t* out;
  uint32_t* scores;       // [tokens][hkv][width], the upper halves of fp64 numbers
  int64_t max_pages;      // the caller's bound of a sequence's pages (0: none)
  int64_t row0, tokens;   // the rows of this launch
  int tiles, run_log;     // blocks along the pages; rows of a block, 1 << run_log
  uint32_t unit0;
};

hipError_t launch_cache_append(const CacheAppend& a, bool bf16, bool e4m3, hipStream_t s);
hipError_t launch_cache_read(const CacheRead& a, bool bf16, bool e4m3, hipStream_t s);
// Fills tile_log, splits and units for at most max_q queries and max_len tokens a
// sequence; returns the workspace bytes.
size_t plan_cache_attn(CacheAttn* a, int64_t max_q, int64_t max_len, size_t* ml_at);
hipError_t launch_cache_attn(const CacheAttn& a, bool bf16, bool e4m3, hipStream_t s);
size_t plan_cache_select(const CacheSelect& a, int64_t* tokens);
hipError_t launch_cache_select(CacheSelect a, bool bf16, hipStream_t s);

inline int cache_width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

}  // namespace rs
