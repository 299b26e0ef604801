"""What the lanes of a wavefront read of a piece of a row, without a GPU: the function that the kernels' loads go by (lane_of_piece), over all lengths of pieces that layouts make."""
import os
import subprocess

import pytest

from conftest import ROOT

PIECES = r"""
#include <stdio.h>
#include "rtopk_draw_shape.hpp"
using namespace rtopk;
constexpr int kRoom = 1 << 15;
static int seen[kRoom];

// Each column of the piece once, none beyond it; batches only of chunks that are there, `some` where a lane has none.
template <int V, int U>
long piece(int cols) {
  long bad = 0;
  if (cols + 64 * V * U > kRoom) return 1;
  for (int c = 0; c < kRoom; ++c) seen[c] = 0;
  for (int lane = 0; lane < 64; ++lane) {
    const auto chunk = [&](int i) {
      for (int c = 0; c < V; ++c) ++seen[i * V + c];
    };
    lane_of_piece<V, U>(
        cols, lane,
        [&](int i) {
          if (U == 1) ++bad;
          for (int u = 0; u < U; ++u) chunk(i + u * 64);
        },
        [&](int i, bool is, bool some) {
          if (is) chunk(i);
          if (!is && !some) ++bad;
        },
        [&](int c) { ++seen[c]; });
  }
  for (int c = 0; c < kRoom; ++c) bad += seen[c] != (c < cols);
  return bad;
}

long pieces(int cols) { return piece<4, 4>(cols) + piece<8, 2>(cols) + piece<4, 1>(cols) + piece<8, 1>(cols); }

int main() {
  long bad = 0;
  for (int cols = 1; cols <= 2100; ++cols) bad += pieces(cols);
  for (int cols = 2100; cols < 20000; cols += 61) bad += pieces(cols);
  for (int k = 1; k < 80; ++k)  // whole numbers of chunks, and one more or fewer of them or of columns
    for (int off = -8; off <= 8; ++off) bad += pieces(k * 256 + off);
  printf("%ld\n", bad);
  return bad != 0;
}
"""


@pytest.mark.parametrize("level", ["-O0", "-O2"])
def test_the_lanes_of_a_piece_read_its_columns_and_no_others(tmp_path, level):
    src = tmp_path / "pieces.cpp"
    src.write_text(PIECES)
    subprocess.check_call(["g++", level, "-std=c++17", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(src), "-o", str(tmp_path / "pieces")])
    out = subprocess.run([str(tmp_path / "pieces")], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
