// How the tiles of dx are shared out.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define STQ_BOTH __host__ __device__
#else
#define STQ_BOTH
#endif

namespace stq {

// The tiles of dx, row by row, and which of `units` (CTAs or pairs) compute what of them.  What is computed together should lie together:
// neighbouring tiles read the same rows of p and the same columns of w, so where the units stand at the same place of their sums, those
// come from memory once.
//
// Whole rounds: unit i has tiles i, i + units, ... as long as there is one for each unit.
// Of the `rest`, as many tiles as there are units for are cut into `parts` equal parts: unit i has part i / cut of tile i % cut.
// What is left then, or all of the rest where parts would be too short, is cut into U equal ranges, one behind the other: unit u has
// [u left / U, (u + 1) left / U) of these tiles.
//
// A part, and what a range has of a tile, is a segment.  Which segments a tile has does not depend on the length of the sums, so every
// piece of the vocabulary adds to the same ones.  They are numbered: parts first, then (r, u) is units + r + u, which no other has.
struct Ranges {
  uint32_t units, tiles_m, tiles, whole, cut, parts, left, U;
  // k: stages of the sum (of the first piece)
  STQ_BOTH Ranges(uint32_t rows, uint32_t tile_m, uint32_t tiles_n, uint32_t k, uint32_t units_) {
    units = units_;
    tiles_m = (rows + tile_m - 1) / tile_m;
    tiles = tiles_m * tiles_n;
    whole = tiles / units * units;
    left = tiles - whole;
    cut = parts = U = 0;
    if (left == 0) return;
    const uint32_t even = units / left;      // parts that leave at most a sixteenth of the units without one, and are not too short
    if (left * even >= units - units / 16 && k >= 4 * even) {
      cut = left;
      parts = even;
    } else {
      const uint32_t more = even + 1, fit = units / more;
      // (four stages to a range at least)
      if ((uint64_t)(left - fit) * k >= 4 * units && k >= 4 * more) {
        cut = fit;
        parts = more;
      }
    }
    left -= cut;
    const uint64_t most = (uint64_t)left * k / (cut ? 8 : 4);      // (next to parts, ranges are short, and every segment is read again)
    U = most < left ? left : most < units ? (uint32_t)most : units;
  }
  // Tile `cut + r` of the rest: r below `left`.  The tiles that range u has something of, and the ranges that tile r is in.
  STQ_BOTH uint32_t tile_first(uint32_t u) const { return u * left / U; }
  STQ_BOTH uint32_t tile_last(uint32_t u) const { return ((u + 1) * left - 1) / U; }
  STQ_BOTH uint32_t first(uint32_t r) const { return r * U / left; }
  STQ_BOTH uint32_t last(uint32_t r) const { return ((r + 1) * U - 1) / left; }
  // Where range u begins in tile r, of k stages (it ends where range u + 1 begins), and where a part does.
  STQ_BOTH uint32_t begin(uint32_t r, uint32_t u, uint32_t k) const {
    const uint32_t at = u * left, from = r * U;
    return at <= from ? 0 : at - from >= U ? k : (uint32_t)((uint64_t)(at - from) * k / U);
  }
  STQ_BOTH uint32_t begin(uint32_t part, uint32_t k) const { return (uint32_t)((uint64_t)part * k / parts); }
  // The segments of a tile of the rest, which follow one another: the first one's number, and how many (r below cut + left).
  STQ_BOTH uint32_t segment(uint32_t r) const { return r < cut ? r * parts : units + r - cut + first(r - cut); }
  STQ_BOTH uint32_t count(uint32_t r) const { return r < cut ? parts : last(r - cut) - first(r - cut) + 1; }
  // All numbers are below this.
  STQ_BOTH static uint32_t segments(uint32_t units) { return 3 * units; }
};

// Blocks of rows to a tile of dx.  Two share each stage of w, three quarters of the bytes of a product, but both accumulators are then one
// tile's, and its results leave while nothing is multiplied.  Two where there is such a tile for every unit at least; with fewer, more and
// smaller tiles leave less to be cut.  dz and dx over 50257 entries, two blocks against one: 8192 x 1600 (112 tiles for 74 pairs) 2059 and
// 2406 us, 4096 x 4096 (128) 2561 and 2543, 6000 x 2560 (120) 2501 and 2436; 8192 x 1024 (64) 1487 and 1437, 4096 x 2048 (64) 1370 and 1367,
// 8192 x 64 (16) 381 and 389.  (Not all of it goes by that: 4096 x 1600, 56 tiles, 1156 and 1255.)  `rows` are those that may count: how
// many do is known on the device alone.
inline int dx_blocks(uint32_t rows, uint32_t block, uint32_t tiles_n, uint32_t units) {
  return (uint64_t)((rows + 2 * block - 1) / (2 * block)) * tiles_n >= units ? 2 : 1;
}

}  // namespace stq
