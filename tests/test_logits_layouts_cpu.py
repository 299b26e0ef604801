"""Rules on how a call's rows are laid over workgroups, swept on the CPU."""
import os
import subprocess

from conftest import ROOT


def run(tmp_path, source):
    """The numbers that a program of the rules' header prints."""
    src, exe = tmp_path / "rules.cpp", tmp_path / "rules"
    src.write_text('#include <stdio.h>\n#include "rtopk_logits_shape.hpp"\nusing namespace rtopk;\n' + source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    return [int(n) for n in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]


FAR = r"""
int main() {
  long bad = 0, grouped = 0;
  const int64_t counts[] = {1, 2, 3, 16, 31, 64, 100, 255, 256, 257, 511, 512, 513, 1000, 4096, 100000, (int64_t)1 << 31};
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int64_t M = 1; M <= kMaxLogitsM; M += M < 20000 ? 7 : M / 97)
      for (int64_t N : counts)
        for (int place = 0; place < 2; ++place) {
          const LogitsLayout l = logits_grad_layout(N, (int)M, dtype, place);
          const int group = far_group(N, l.segments);
          if (group < 1 || group > l.segments) ++bad;
          grouped += group > 1;
          // the workgroups that read a row whole: four at most, or one to a row, or as many as fill the GPU twice (each row's last group is a partial one)
          const int64_t reading = ceil_div(l.segments, group);
          if (reading > 4 && N * (reading - 1) > 512) ++bad;
          if (place && reading != 1) ++bad;
        }
  printf("%ld %ld\n", bad, grouped);
  return 0;
}
"""


def test_workgroups_that_take_a_rows_sums_again(tmp_path):
    """Their number does not grow with the row's width once rows fill the GPU: what is read again is at most 4 times the rows, or 512 rows."""
    bad, grouped = run(tmp_path, FAR)
    assert bad == 0 and grouped > 0
