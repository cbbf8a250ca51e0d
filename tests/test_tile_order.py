"""The order in which the blocks of a block-scaled product take its tiles (csrc/tile_order.h), walked through on the host: every tile once, whatever the
launch's size (no GPU needed)."""
import ctypes
import shutil
import subprocess

import numpy as np
import pytest

from paper_2502_02581_amd import build

SHIM = r"""
#include "tile_order.h"
using namespace moe;
// how often each tile [mt][nt] is taken by the blocks of a launch with room for `room` tiles; -1: a place that is no tile
extern "C" int planned(int n_mt, int ntn, int room, int from_back, int* taken) {
  const int total = n_mt * ntn, blocks = (room + 255) / 256 * 256;
  for (int b = 0; b < blocks; b++) {
    const int q = dealt_tile(b, total);
    if (q >= total) continue;
    const TilePlace t = band_tile(q, n_mt, ntn, from_back);
    if (q < 0 || t.mt < 0 || t.mt >= n_mt || t.nt < 0 || t.nt >= ntn) return -1;
    taken[t.mt * ntn + t.nt]++;
  }
  return 0;
}
// the same of pieces: [mt][piece][nt], `tail` of them a tile; a whole tile takes all of its own
extern "C" int cut(int n_mt, int ntn, int tail, int* taken) {
  const int total = n_mt * ntn, blocks = cut_tile_blocks(total, tail);
  for (int b = 0; b < blocks; b++) {
    const CutTile c = cut_tile(b, total, tail);
    if (c.q >= total) continue;
    const TilePlace t = band_tile(c.q, n_mt, ntn, 0);
    if (c.q < 0 || t.mt < 0 || t.mt >= n_mt || t.nt < 0 || t.nt >= ntn || c.piece < 0 || c.piece >= c.pieces) return -1;
    if (c.pieces != 1 && c.pieces != tail) return -1;
    for (int i = 0; i < tail; i++)
      if (c.pieces == 1 || i == c.piece) taken[(t.mt * tail + i) * ntn + t.nt]++;
  }
  return 0;
}
extern "C" int dealt(int block, int total) { return dealt_tile(block, total); }
"""


@pytest.fixture(scope="module")
def order(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("order")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    return ctypes.CDLL(str(d / "shim.so"))


# up to twelve rounds: below and beyond the four from which bands come from both ends and the six beyond which runs are long; bands of one to four rows
SIZES = [(m, n) for n in (1, 2, 3, 5, 8, 11, 16, 28, 50) for m in (1, 2, 3, 4, 5, 7, 8, 15, 31, 64, 65, 86, 97, 129, 256, 259, 515, 1030, 2050) if m * n <= 3200]


def count(n):
    a = np.zeros(n, np.int32)
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int))


@pytest.mark.parametrize("room", [1, 3])   # a plan may have fewer tiles than the launch has room for
def test_every_tile_once(order, room):
    rounds = set()
    for n_mt, ntn in SIZES:
        total = n_mt * ntn
        rounds.add(total >> 8)
        for back in {0, n_mt // 4 // 3 if total >> 8 >= 4 else 0}:
            taken, p = count(total)
            assert order.planned(n_mt, ntn, room * total, back, p) == 0, (n_mt, ntn, back)
            assert (taken == 1).all(), (n_mt, ntn, back)
    assert {0, 3, 4, 6, 7, 8, 11, 12} <= rounds


@pytest.mark.parametrize("tail", [1, 2, 4])
def test_every_piece_once(order, tail):
    for n_mt, ntn in SIZES:
        taken, p = count(n_mt * ntn * tail)
        assert order.cut(n_mt, ntn, tail, p) == 0 and (taken == 1).all(), (n_mt, ntn)


def test_runs_of_an_xcd(order):
    """Blocks go round the eight XCDs; of a full round each takes runs of 8 consecutive tiles, in all but the last round of long launches one run of 32."""
    for rounds in (1, 6, 7, 9):
        for r in range(rounds):
            for xcd in range(8):
                tiles = [order.dealt(r * 256 + i * 8 + xcd, rounds * 256 + 17) - r * 256 for i in range(32)]
                run = 32 if rounds > 6 and r < rounds - 1 else 8
                starts = tiles[::run]
                assert tiles == [s + i for s in starts for i in range(run)] and all(s % run == 0 and 0 <= s < 256 for s in starts)
