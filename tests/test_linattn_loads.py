"""Addresses of linear attention's tile loads (csrc/seq_internal.h, lin_piece), enumerated on the CPU for every width, both
types and every tile: no lane loads from outside its row, every element of a tile gets to its place in LDS, and what is
behind a row's end there is left alone."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <stdio.h>
#include <vector>
#include "seq_internal.h"
using namespace pnn;

// a tile of W columns, `width` elements from its first one to the row's end and `before` in front of it; LDS rows have
// `pad` pieces more than they need, and one piece is in front of the first
int tile(int ve, int threads, int W, int pad, int width, int before) {
  const int rows = LIN_CHUNK, pieces = W / ve, loads = (rows * pieces + threads - 1) / threads, apart = threads / pieces;
  const int LD = W + pad * ve, size = ve + rows * LD;
  std::vector<int> lds(size, -1);
  for (int lane = 0; lane < threads; ++lane) {
    const LinPiece x = lin_piece(lane, rows, pieces, ve, width);
    for (int j = 0; j < loads; ++j) {
      const int row = x.row + j * apart, at = ve + row * LD + x.to;
      if (row < 0 || row >= rows) return printf("row %d\n", row), 1;
      if (x.from < -before || x.from + ve > width)
        return printf("%d + %d of a row from %d to %d\n", x.from, ve, -before, width), 1;
      if (at < 0 || at + ve > size) return printf("LDS %d of %d\n", at, size), 1;
      for (int e = 0; e < ve; ++e) lds[at + e] = row * 1000 + x.from + e + 256;
    }
  }
  for (int row = 0; row < rows; ++row)
    for (int c = 0; c < W; ++c) {
      const int got = lds[ve + row * LD + c], want = c < width ? row * 1000 + c + 256 : -1;
      if (got != want) return printf("LDS row %d column %d: %d for %d\n", row, c, got, want), 1;
    }
  return 0;
}

int main() {
  long tiles = 0;
  for (int size = 2; size <= 4; size += 2)
    for (int waves = 4; waves <= 8; waves += 4)
      for (int width = 16 / size; width <= LIN_MAX_WIDTH; ++width) {
        const int ve = 16 / size, threads = 64 * waves;
        for (int pad = 64; pad <= 256; pad *= 2)       // queries and keys, whole rows
          for (int more = 2; more <= 4; more += 2)
            if (width <= pad && ++tiles && tile(ve, threads, pad, more, width, 0))
              return printf("inner: size %d waves %d pad %d width %d\n", size, waves, pad, width), 1;
        const int W = 16 * waves;                      // values, a block of columns
        for (int block = 0; block * W < width; ++block)
          if (++tiles && tile(ve, threads, W, 2, width - block * W, block * W))
            return printf("values: size %d waves %d width %d block %d\n", size, waves, width, block), 1;
      }
  printf("%ld tiles\n", tiles);
  return 0;
}
"""


def test_every_piece_is_in_its_row(tmp_path):
    src, exe = tmp_path / "loads.cpp", tmp_path / "loads"
    src.write_text(SOURCE)
    r = subprocess.run(["hipcc", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-std=c++17", "-O1", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2103_08802_amd", "csrc"),
                        str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout.split()[0]) > 2000
