"""How the tiles of dx are shared out (stq_vocab_ranges.h), over all small cases and at random large ones (no GPU)."""
import ctypes as C
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2604_06836_b200", "csrc")

SOURCE = r"""
#include <vector>
#include "stq_vocab_ranges.h"
using stq::Ranges;
// 0: the ranges are what they have to be; else which rule is broken.  k: stages of the first piece, later: of another one.
extern "C" int check(uint32_t rows, uint32_t tile_m, uint32_t tiles_n, uint32_t k, uint32_t later, uint32_t units) {
  const Ranges r(rows, tile_m, tiles_n, k, units);
  if (r.tiles_m != (rows + tile_m - 1) / tile_m || r.tiles != r.tiles_m * tiles_n) return 1;
  if (r.whole % units || r.whole + r.rest != r.tiles || r.rest >= units) return 2;
  if (r.rest == 0) return 0;
  if (r.U < r.rest || r.U > units || (r.split && r.U != r.split * r.rest)) return 3;
  std::vector<char> taken(r.U), used(Ranges::segments(units));
  for (uint32_t i = 0; i < r.U; ++i) {
    if (r.unit(i) >= r.U || taken[r.unit(i)]++) return 4;                    // some range twice
  }
  std::vector<uint64_t> length(r.U);
  for (uint32_t t = 0; t < r.rest; ++t) {
    if (r.first(t) > r.last(t) || r.last(t) >= r.U) return 5;
    for (int pass = 0; pass < 2; ++pass) {
      const uint32_t kk = pass ? later : k;
      uint32_t at = 0;
      for (uint32_t u = r.first(t); u <= r.last(t); ++u) {
        const uint32_t b = r.begin(t, u, kk), e = r.begin(t, u + 1, kk);
        if (b != at || e < b || e > kk) return 6;                            // a gap, or twice
        if (t < r.tile_first(u) || t > r.tile_last(u)) return 7;
        if (pass == 0) {
          length[u] += e - b;
          if (t + u >= used.size() || used[t + u]++) return 8;               // two segments with one number
        }
        at = e;
      }
      if (at != kk) return 9;                                                // not the whole sum
    }
  }
  uint64_t least = ~0ull, most = 0;
  for (uint32_t u = 0; u < r.U; ++u) {
    for (uint32_t t = r.tile_first(u); t <= r.tile_last(u); ++t)
      if (u < r.first(t) || u > r.last(t)) return 10;                        // the two views differ
    least = length[u] < least ? length[u] : least;
    most = length[u] > most ? length[u] : most;
  }
  return most - least > 2 ? 11 : 0;                                          // not balanced
}
"""


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    at = tmp_path_factory.mktemp("ranges")
    src, lib = at / "ranges.cpp", at / "ranges.so"
    src.write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", CSRC, "-shared", "-fPIC", "-o", str(lib), str(src)])
    f = C.CDLL(str(lib)).check
    f.argtypes = [C.c_uint32] * 6
    return f


def test_small(check):
    for tiles_m in range(0, 7):
        for tiles_n in (1, 2, 3, 7, 13):
            for k in (1, 2, 3, 4, 5, 7, 8, 13, 40):
                for units in (1, 2, 3, 5, 8, 16, 74, 148):
                    for later in (1, k, max(1, k - 1)):
                        case = (tiles_m * 128, 128, tiles_n, k, later, units)
                        assert check(*case) == 0, case


def test_large(check):
    rng = random.Random(1)
    for _ in range(5000):
        cg = rng.choice((1, 2))
        tile_m = 128 * cg * (rng.choice((1, 2)) if cg == 2 else 1)
        rows = rng.choice((1, 100, 128)) if cg == 1 else rng.randint(1, 262144)
        k = rng.randint(1, 262144)
        case = (rows, tile_m, rng.randint(1, 512), k, rng.randint(1, k), 148 // cg)
        assert check(*case) == 0, case
