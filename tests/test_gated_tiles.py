"""The gated block's mapping of blocks to tiles, from the kernels' own header, compiled for the host."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2212_11142_amd", "csrc")
PROGRAM = r"""
#include "gated_tiles.h"
#include <cstdio>
#include <cstdlib>
int main(int, char **v) {
  const int nm = std::atoi(v[1]), nn = std::atoi(v[2]);
  for (unsigned b = 0; b < (unsigned)(nm * nn); ++b) {
    const bgp::Tile t = bgp::tile_of(b, nm * nn, nm, nn);
    std::printf("%d %d\n", t.m, t.n);
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    src, exe = d / "t.cpp", d / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + CSRC, str(src), "-o", str(exe)], check=True)
    return str(exe)


@pytest.mark.parametrize("nm,nn", [(1, 1), (3, 5), (8, 4), (9, 7), (64, 32), (17, 1), (1, 40), (512, 16), (5, 63)])
def test_every_tile_has_its_block(program, nm, nn):
    out = subprocess.run([program, str(nm), str(nn)], capture_output=True, text=True, check=True, timeout=60).stdout
    tiles = [tuple(map(int, line.split())) for line in out.split("\n") if line]
    assert len(tiles) == nm * nn and set(tiles) == {(m, n) for m in range(nm) for n in range(nn)}
    # an XCD's blocks, every eighth, go through eight tiles of m or fewer at a time, one n after the other
    for x in range(8):
        mine = tiles[x::8]
        for a, b in zip(mine, mine[1:]):
            assert b[0] // 8 > a[0] // 8 or (b[0] // 8 == a[0] // 8 and (b[1], b[0]) > (a[1], a[0]))


def test_the_kernels_have_no_other():
    assert "Tile tile_of(" not in open(os.path.join(CSRC, "gated.hip")).read()
