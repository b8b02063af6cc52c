// The tiles of query rows that a launch of the page scores takes (host arithmetic only).
//
// A tile is 1 << log rows of a sequence. Tile numbers, as the kernels find them: padded,
// ceil(pad / run) a sequence; packed, sequence s from (off[s] >> log) + s on, s alone left
// out where log is 0, as single rows never end within a tile.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace rs {

struct TileRange {
  int64_t first, count;
};

// The tiles that rows [row0, row0 + n) may lie in. Packed, the host does not know the
// offsets: a row's tile is from (row >> log) - 1 on, and at most seqs - 1 past row >> log.
inline TileRange tiles_of_rows(int64_t seqs, int64_t rows, int64_t pad, int log, int64_t row0, int64_t n) {
  const int64_t run = int64_t(1) << log;
  if (pad > 0) {
    const int64_t per = (pad + run - 1) >> log, last = row0 + n - 1;
    const int64_t first = row0 / pad * per + (row0 % pad >> log);
    return {first, last / pad * per + (last % pad >> log) + 1 - first};
  }
  if (log == 0) return {row0, n};
  const int64_t first = std::max(int64_t(0), (row0 >> log) - 1);
  const int64_t end = std::min((rows >> log) + seqs, ((row0 + n - 1) >> log) + seqs);
  return {first, end - first};
}

// Rows of a tile, as a power of two: about those of a sequence, and at most `most`. Where
// the rows are taken `window` at a time, packed sequences cost every window a tile each
// beside its rows: single rows then, where those are the more.
inline int tile_rows_log(int64_t seqs, int64_t rows, int64_t pad, int64_t window, int64_t most) {
  int log = 0;
  while ((int64_t(2) << log) <= rows / seqs && (int64_t(2) << log) <= most) ++log;
  return window < rows && pad == 0 && seqs > window >> log ? 0 : log;
}

}  // namespace rs
