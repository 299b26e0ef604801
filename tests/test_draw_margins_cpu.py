"""The margins that drafts are tested with in fp32, without a GPU: wider than what two rows' sums may be off by, for every row and workgroup that tests them."""
import os
import subprocess

from conftest import ROOT

MARGINS = r"""
#include <stdio.h>
#include "rtopk_draw_shape.hpp"
using namespace rtopk;
int main() {
  long bad = 0, most[2] = {0, 0};
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int M = 1; M <= kMostTested; M += M < kMostTested - 500 ? 499 : 1)
      for (int waves = 4; waves <= 16; waves *= 2)
        for (int far = 0; far < 2; ++far) {
          const int64_t units = test_units(M, dtype, waves, far);
          most[far] = units > most[far] ? units : most[far];
          // u q and p are each off by `units`, and by the square of that in the second order
          const double off = 2.0 * units * 0x1p-24;
          if (off + off * off >= (far ? kFarTestMargin : kTestMargin)) ++bad;
          // no fewer than the additions to a thread's sum, one behind the other
          const int64_t columns = (M + 64 * waves - 1) / (64 * waves), each = logits_width(dtype) * test_loads(waves);
          if (units < (far ? columns : columns / each)) ++bad;
        }
  printf("%ld bad, at most %ld units, far %ld\n", bad, most[0], most[1]);
  return bad != 0;
}
"""


def test_margins(tmp_path):
    src = tmp_path / "margins.cpp"
    src.write_text(MARGINS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(src), "-o", str(tmp_path / "margins")])
    out = subprocess.run([str(tmp_path / "margins")], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
