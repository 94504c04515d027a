"""The order in which a windowed decode step over pages takes a head's tiles (csrc/tile_order.h), compiled for the host: every tile
has one place, and a place without a tile is told from those with one by its first row, up to the longest head there is."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_09754_amd", "csrc")

ORDER = r"""
#include <cstdio>
#include <initializer_list>
#include <vector>
#include "tile_order.h"
using namespace lava;
int main() {
  long long beyond = 0;
  std::vector<long long> lengths;
  for (int rows = 1; rows < 80 * kTileKeys; rows += 7) lengths.push_back(rows);
  for (long long page : {16, 32, 64, 128, 256})
    for (long long back = 1; back <= 640; back += 31) lengths.push_back((1ll << 31) - page - 16 * (back - 1));
  for (long long rows : lengths) {
    const int tiles = (int)((rows + kTileKeys - 1) / kTileKeys);
    const int columns = spread_columns(tiles, true), places = places_of(tiles, true);
    if (places < tiles || places >= tiles + kSpread) return 1;
    // of a long head the places at both ends of every matrix row, where a tile may be missing
    std::vector<int> seen(rows < 100000 ? tiles : 0);
    for (int x = 0; x < places; ++x) {
      if (rows >= 100000 && x >= 3 * kSpread && x < places - 3 * kSpread) x = places - 3 * kSpread;
      const long long tile = columns > 0 ? (long long)(x % kSpread * kStep % kSpread) * columns + x / kSpread : x;
      const bool there = tile < tiles;
      if ((row_at(x, columns) < (unsigned)rows) != there) {
        std::printf("%lld rows: place %d is tile %lld, first row %u\n", rows, x, tile, row_at(x, columns));
        return 2;
      }
      if (there && row_at(x, columns) != (unsigned)(tile * kTileKeys)) return 3;
      if (tile * kTileKeys > 0x7fffffffll) ++beyond;
      if (there && rows < 100000 && seen[tile]++) return 4;
    }
    for (int n : seen)
      if (n != 1) return 5;
  }
  std::printf("%lld\n", beyond);
  return 0;
}
"""


def test_every_tile_has_one_place(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(ORDER)
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", CSRC,
                    str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
    assert int(res.stdout) > 0                                      # places whose first row passes 31 bits were among them
