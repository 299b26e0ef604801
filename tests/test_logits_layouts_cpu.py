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


KERNELS = r"""
int main() {
  // rows by one workgroup at 97 rows, and the (wavefronts, loads) that hold them; columns of fp32, twice as many in 16 bits
  const int columns[] = {256, 257, 1024, 4096, 4097, 8192, 8193, 16384, 16385, 32768, 32769, 49152, 49157, 65536, 65541};
  for (int dtype = 0; dtype < 3; dtype += 2)
    for (int M : columns) {
      M = dtype == 0 ? M : 2 * M;
      const HeldLayout h = held_layout(M, dtype);
      printf("%d %d %d\n", logits_layout(97, M, dtype, 0).segments, h.waves, h.loads);
    }
  // the lines of the spread rows: segments with scratch memory
  const int64_t calls[][4] = {{2, 32768, 0, 0}, {2, 32769, 0, 0}, {95, 32769, 0, 32}, {95, 32769, 0, 33}, {96, 32769, 0, 0}, {2, 65537, 2, 32}, {2, 65536, 2, 32}, {3, 262144, 0, 20}, {1, 1 << 20, 1, 9}};
  for (const auto& c : calls) printf("%d\n", logits_layout(c[0], (int)c[1], (int)c[2], (int)c[3]).segments);
  return 0;
}
"""


def test_which_kernel_takes_a_row(tmp_path):
    """The widths of the GPU tests reach the kernels that they are meant for."""
    n = run(tmp_path, KERNELS)
    rows = [tuple(n[3 * i:3 * i + 3]) for i in range(30)]
    narrow = [(1, 1, 4)] * 3 + [(1, 4, 4)] * 2 + [(1, 4, 8)] * 2 + [(1, 8, 8)] * 2 + [(1, 8, 16)] * 2 + [(1, 8, 24)]
    read_twice = (1, 8, 0)
    assert rows[:15] == narrow + [(1, 16, 16)] * 2 + [read_twice]
    assert rows[15:] == narrow + [(1, 8, 32)] * 2 + [read_twice]
    assert n[90:] == [1, 9, 9, 1, 1, 9, 1, 64, 128]


REACHED = r"""
int main() {
  // every kernel that is compiled for a type is some width's, and every width's is compiled
  int bad = 0, kernels = 0;
  for (int dtype = 0; dtype < 3; ++dtype) {
#define X(w, r, q)                                            \
  {                                                           \
    bool found = false;                                       \
    for (int M = 1; M <= 200000; ++M) {                       \
      const HeldLayout h = held_layout(M, dtype);             \
      found |= h.waves == w && h.loads == r + q;              \
    }                                                         \
    bad += found != is_held_by(dtype, w, r);                  \
    kernels += found;                                         \
  }
    RTOPK_HELD_LIST(X)
  }
  printf("%d %d\n", bad, kernels);
  return 0;
}
"""


def test_every_kernel_that_holds_a_row_is_reached(tmp_path):
    assert run(tmp_path, REACHED) == [0, 21]
