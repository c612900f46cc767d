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
  const uint32_t rest = r.tiles - r.whole;
  if (r.tiles_m != (rows + tile_m - 1) / tile_m || r.tiles != r.tiles_m * tiles_n) return 1;
  if (r.whole % units || r.whole > r.tiles || rest >= units || r.cut + r.left != rest) return 2;
  if (r.cut && (r.parts < 1 || r.cut * r.parts > units || k < 4 * r.parts)) return 3;
  std::vector<char> used(Ranges::segments(units));
  std::vector<uint64_t> length(units);
  for (uint32_t t = 0; t < rest; ++t)
    for (uint32_t i = 0; i < r.count(t); ++i) {
      if (r.segment(t) + i >= used.size() || used[r.segment(t) + i]++) return 4;      // a number that two have
    }
  for (int pass = 0; pass < 2; ++pass) {
    const uint32_t kk = pass ? later : k;
    for (uint32_t t = 0; t < r.cut; ++t) {
      uint32_t at = 0;
      for (uint32_t p = 0; p < r.parts; ++p) {
        if (r.begin(p, kk) != at || r.begin(p + 1, kk) < at) return 5;
        at = r.begin(p + 1, kk);
        if (!pass) length[p * r.cut + t] += at - r.begin(p, kk);
      }
      if (at != kk) return 6;
    }
    if (r.left && (r.U < r.left || r.U > units)) return 7;
    for (uint32_t t = 0; t < r.left; ++t) {
      if (r.first(t) > r.last(t) || r.last(t) >= r.U) return 8;
      uint32_t at = 0;
      for (uint32_t u = r.first(t); u <= r.last(t); ++u) {
        const uint32_t b = r.begin(t, u, kk), e = r.begin(t, u + 1, kk);
        if (b != at || e < b || e > kk) return 9;                            // a gap, or twice
        if (t < r.tile_first(u) || t > r.tile_last(u)) return 10;
        if (r.segment(r.cut + t) + u - r.first(t) != units + t + u) return 11;
        if (!pass) length[u] += e - b;
        at = e;
      }
      if (at != kk) return 12;                                               // not the whole sum
    }
  }
  for (uint32_t u = 0; r.left && u < r.U; ++u)
    for (uint32_t t = r.tile_first(u); t <= r.tile_last(u); ++t)
      if (t >= r.left || u < r.first(t) || u > r.last(t)) return 13;         // the two views differ
  uint64_t most = 0;
  for (uint64_t l : length) most = l > most ? l : most;
  // no unit has much more than its share: an eighth, the roundings, and what comes of ranges of eight stages at least
  return most > (uint64_t)rest * k / units * 9 / 8 + 12 ? 14 : 0;
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
