"""Rules by which the vocabulary gradients choose their tiles (no GPU)."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_06836_b200", "csrc")
SOURCE = """
#include "stq_vocab_ranges.h"
extern "C" int blocks(uint32_t rows, uint32_t block, uint32_t tiles_n, uint32_t units) { return stq::dx_blocks(rows, block, tiles_n, units); }
"""


@pytest.fixture(scope="module")
def blocks(tmp_path_factory):
    at = tmp_path_factory.mktemp("rules")
    (at / "rules.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", CSRC, "-shared", "-fPIC", "-o", str(at / "rules.so"), str(at / "rules.cpp")])
    f = C.CDLL(str(at / "rules.so")).blocks
    f.argtypes = [C.c_uint32] * 4
    return f


def test_two_blocks_of_rows_go_by_tiles(blocks):
    """Not by tokens: few columns make few tiles of any number of tokens, many columns make enough of few."""
    assert blocks(8192, 256, 1, 74) == 1 and blocks(4096, 256, 16, 74) == 2
    for units in (2, 74, 80):
        for tiles_n in (1, 3, 7, 32, 256):
            for rows in range(256, 20000, 256):
                tiles = -(-rows // 512) * tiles_n
                assert blocks(rows, 256, tiles_n, units) == (2 if tiles >= units else 1)
    assert blocks(262144, 256, 512, 74) == 2
