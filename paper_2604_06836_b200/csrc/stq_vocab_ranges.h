// How the tiles of dx are shared out.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define STQ_BOTH __host__ __device__
#else
#define STQ_BOTH
#endif

namespace stq {

// The tiles of dx, row by row, and which of `units` (CTAs or pairs) compute what of them.
//
// Whole rounds: unit i has tiles i, i + units, ... as long as there is one for each unit.  All units then stand at the same place of their
// sums, and what neighbouring tiles read (rows of p, columns of w) comes from memory once.
// The `rest` tiles that are left are cut into U equal ranges, one behind the other: unit u has [u rest / U, (u + 1) rest / U) of them.
// What a range has of a tile is a segment; tile r has the segments of units first(r) .. last(r), whatever the length of the sums, so
// that every piece of the vocabulary adds to the same segments.  Segment (r, u) has number r + u, which no other has.
struct Ranges {
  uint32_t tiles_m, tiles, whole, rest, U, split;
  // k: stages of the sum (of the first piece)
  STQ_BOTH Ranges(uint32_t rows, uint32_t tile_m, uint32_t tiles_n, uint32_t k, uint32_t units) {
    tiles_m = (rows + tile_m - 1) / tile_m;
    tiles = tiles_m * tiles_n;
    whole = tiles / units * units;
    rest = tiles - whole;
    const uint64_t most = (uint64_t)rest * k / 4;      // (four stages to a range at least)
    U = most < rest ? rest : most < units ? (uint32_t)most : units;
    // few tiles: every tile in as many ranges, if that leaves no more than a sixteenth of the units without one.  Then those that have
    // the same share of a row of tiles run side by side, and read whole rows of w together.
    const uint32_t even = rest && U > rest ? U / rest * rest : 0;
    split = even && U - even <= U / 16 ? even / rest : 0;
    if (split) U = even;
  }
  // The range that the i-th CTA or pair takes (i < U).
  STQ_BOTH uint32_t unit(uint32_t i) const { return split ? i % rest * split + i / rest : i; }
  // The tiles of the rest that range u has something of, and the ranges that tile r is in.
  STQ_BOTH uint32_t tile_first(uint32_t u) const { return u * rest / U; }
  STQ_BOTH uint32_t tile_last(uint32_t u) const { return ((u + 1) * rest - 1) / U; }
  STQ_BOTH uint32_t first(uint32_t r) const { return r * U / rest; }
  STQ_BOTH uint32_t last(uint32_t r) const { return ((r + 1) * U - 1) / rest; }
  // Where range u begins in tile r, of k stages; it ends where range u + 1 begins.
  STQ_BOTH uint32_t begin(uint32_t r, uint32_t u, uint32_t k) const {
    const uint32_t at = u * rest, from = r * U;
    return at <= from ? 0 : at - from >= U ? k : (uint32_t)((uint64_t)(at - from) * k / U);
  }
  // Segments have numbers below this.
  STQ_BOTH static uint32_t segments(uint32_t units) { return 2 * units; }
};

}  // namespace stq
