// How the sums of the tiles of dx are shared out.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define STQ_BOTH __host__ __device__
#else
#define STQ_BOTH
#endif

namespace stq {

// Tiles of dx, row by row, and which units (CTAs or pairs) add to which: unit u has stages [u S / U, (u + 1) S / U) of the S = tiles * ksteps.
struct Ranges {
  uint32_t tiles_m, tiles, ksteps, U, split;
  uint64_t S;
  STQ_BOTH Ranges(uint32_t rows, uint32_t tile_m, uint32_t tiles_n, uint32_t k, uint32_t units, uint32_t plane_rows) {
    tiles_m = (rows + tile_m - 1) / tile_m;
    tiles = tiles_m * tiles_n;
    ksteps = k;
    S = (uint64_t)tiles * k;
    U = split = 0;
    if (S == 0) return;
    // so long a range that no tile has more units than there are planes
    const uint32_t planes = plane_rows / (tiles_m * tile_m), least = planes > 2 ? (k + planes - 2) / (planes - 1) : k;
    const uint64_t most = ratio(S, least);
    U = (uint32_t)(units < most ? units : most);
    // few tiles: every tile in as many ranges, if that leaves no more than a sixteenth of the units without one.  Then those that have
    // the same share of a row of tiles run side by side, and read whole rows of w together.
    const uint32_t even = U > tiles ? U / tiles * tiles : 0;
    split = even && U - even <= U / 16 ? even / tiles : 0;
    if (split) U = even;
  }
  // The unit whose range the i-th CTA or pair takes.
  STQ_BOTH uint32_t unit(uint32_t i) const { return split ? i % tiles * split + i / tiles : i; }
  STQ_BOTH uint64_t begin(uint32_t u) const { return ratio(u * S, U); }
  STQ_BOTH uint32_t unit_of(uint64_t s) const { return (uint32_t)ratio((s + 1) * U - 1, S); }
  // (a division of 64 bits takes a GPU ten times as long)
  STQ_BOTH static uint64_t ratio(uint64_t a, uint64_t b) { return (a | b) >> 32 ? a / b : (uint32_t)a / (uint32_t)b; }
  // Tile number q of the order that the ranges are cut in.  A unit has r tiles or so, one after the other: they are chosen so that at any
  // time the units' tiles are neighbours (whole rows of tiles, which read the same rows of p).
  STQ_BOTH uint32_t tile(uint32_t q) const {
    const uint32_t r = tiles / U, c = r > 1 ? tiles / r : 0;
    return q < r * c ? q % r * c + q / r : q;
  }
  STQ_BOTH uint32_t place(uint32_t tile) const {      // (its inverse)
    const uint32_t r = tiles / U, c = r > 1 ? tiles / r : 0;
    return tile < r * c ? tile % c * r + tile / c : tile;
  }
  STQ_BOTH uint32_t shares(uint32_t tile) const {
    const uint64_t at = (uint64_t)place(tile) * ksteps;
    return unit_of(at + ksteps - 1) - unit_of(at) + 1;
  }
};

}  // namespace stq
