"""How the sums of the tiles of dx are shared out (stq_vocab_ranges.h), over all small cases and at random large ones (no GPU)."""
import ctypes as C
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2604_06836_b200", "csrc")

SOURCE = r"""
#include <stdio.h>
#include "stq_vocab_ranges.h"
using stq::Ranges;
// 0: the ranges are what they have to be; else which rule is broken.
extern "C" int check(uint32_t rows, uint32_t tile_m, uint32_t tiles_n, uint32_t k, uint32_t units, uint32_t plane_rows) {
  const Ranges r(rows, tile_m, tiles_n, k, units, plane_rows);
  if (r.tiles == 0) return r.U == 0 ? 0 : 1;
  if (r.U == 0 || r.U > units) return 2;
  if (r.begin(0) != 0 || r.begin(r.U) != r.S) return 3;
  const uint32_t planes = plane_rows / (r.tiles_m * tile_m);
  if (r.split && r.U != r.split * r.tiles) return 10;
  uint64_t longest = 0, shortest = ~0ull, units_seen = 0;
  for (uint32_t i = 0; i < r.U; ++i) {
    if (r.unit(i) >= r.U) return 11;
    units_seen += r.unit(i);
  }
  if (units_seen != (uint64_t)r.U * (r.U - 1) / 2) return 12;                // some unit twice
  for (uint32_t u = 0; u < r.U; ++u) {
    const uint64_t b = r.begin(u), e = r.begin(u + 1);
    if (e <= b) return 4;                                                    // nothing to do
    if (r.unit_of(b) != u || r.unit_of(e - 1) != u) return 5;
    longest = e - b > longest ? e - b : longest;
    shortest = e - b < shortest ? e - b : shortest;
  }
  if (longest - shortest > 1) return 6;
  for (uint32_t q = 0; q < r.tiles; ++q) {
    const uint32_t tile = r.tile(q);
    if (tile >= r.tiles || r.place(tile) != q) return 9;                     // not a permutation
    const uint32_t t = q, n = r.shares(tile), first = r.unit_of((uint64_t)t * k);
    if (n == 0 || n > planes) return 7;                                      // more than there are planes for
    uint32_t seen = 0;
    for (uint32_t u = first; u < r.U && r.begin(u) < (uint64_t)(t + 1) * k; ++u) seen += r.begin(u + 1) > (uint64_t)t * k;
    if (seen != n) return 8;
  }
  return 0;
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
    for tiles_m in range(0, 5):
        for tiles_n in (1, 2, 3, 7):
            for k in range(1, 14):
                for units in (1, 2, 3, 5, 8, 74):
                    for planes in (2, 3, 4, 5, 9):
                        case = (tiles_m * 128, 128, tiles_n, k, units, planes * max(1, tiles_m) * 128)
                        assert check(*case) == 0, case


def test_large(check):
    rng = random.Random(1)
    for _ in range(2000):
        cg = rng.choice((1, 2))
        rows = rng.choice((1, 100, 128)) if cg == 1 else rng.randint(1, 16384)
        d = rng.randint(1, 65536)
        ldd = (d + 31) // 32 * 32
        most = 128 if cg == 1 else (rng.randint(rows, 16384 + rows) + 255) // 256 * 256
        plane_rows = max(2 * most, (16 << 20) // ldd)
        tiles_n = -(-d // (128 * cg))
        case = (rows, 128 * cg, tiles_n, rng.randint(1, 2048), 148 // cg, plane_rows)
        assert check(*case) == 0, case
