"""A router's balance loss without a GPU: arguments refused on the host, the layout of every call, and the definitions themselves (oracle/balance.py)
against differences."""
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT
from oracle import balance as definition


@pytest.fixture(scope="module")
def lib():
    import paper_2409_00822_amd as R

    if not os.path.exists(R.lib_path()):
        from paper_2409_00822_amd import build

        build.build()
    return R.load_library()


P = [1 << 30, 1 << 32, 1 << 34, 1 << 36, 1 << 38, 1 << 40, 1 << 42, 1 << 44]  # far apart, aligned, never dereferenced
F32, F16, BF16 = 0, 1, 2


def test_refusals(lib):
    def loss(x=P[0], dtype=F32, N=40, E=16, stride=16, cols=P[1], col_bytes=4, k=2, groups=4, out=P[2], z=P[3], probs=P[4], counts=P[5], rows=P[6], ws=None, n=0):
        return lib.rtopk_balance_loss(x, dtype, N, E, stride, cols, col_bytes, k, groups, out, z, probs, counts, rows, ws, n, None)

    def grad(g=P[2], gz=None, gv=None, x=P[0], dtype=F32, N=40, E=16, stride=16, cols=P[1], col_bytes=4, k=2, groups=4, counts=P[3], rows=P[4], dx=P[5], ds=16):
        return lib.rtopk_balance_loss_backward(g, gz, gv, x, dtype, N, E, stride, cols, col_bytes, k, groups, counts, rows, dx, ds, None)

    for f in (loss, grad):
        for kw in (dict(x=None), dict(cols=None), dict(counts=None), dict(rows=None)):
            assert f(**kw) == -1, (f, kw)
        for kw in (dict(N=-4), dict(E=0), dict(k=0), dict(k=17), dict(groups=0), dict(groups=3), dict(groups=(1 << 20) + 1, N=(1 << 20) + 1), dict(stride=15), dict(stride=2**62),
                   dict(N=2**40), dict(N=2**62)):
            assert f(**kw) == -2, (f, kw)
        assert f(E=1025, stride=1025) == -4 and f(E=257, stride=257, col_bytes=1) == -4
        for kw in (dict(dtype=3), dict(col_bytes=2), dict(col_bytes=8)):
            assert f(**kw) == -10, (f, kw)
        for kw in (dict(x=P[0] + 2), dict(cols=P[1] + 2), dict(counts=P[5] + 1), dict(rows=P[6] + 2), dict(dtype=BF16, x=P[0] + 1)):
            assert f(**kw) == -5, (f, kw)
    assert loss(out=None) == -1 and loss(n=-1) == -2 and loss(k=16, N=4 * (2**31 - 4)) == -2
    for kw in (dict(out=P[0]), dict(z=P[2] + 12), dict(probs=P[1] + 316), dict(counts=P[4] + 252), dict(rows=P[0] + 2556), dict(ws=P[0], n=64)):
        assert loss(**kw) == -8, kw
    assert loss(ws=P[7] + 8, n=64) == -5
    assert grad(N=0) == 0 and grad(g=None) == -1 and grad(dx=None) == -1 and grad(ds=15) == -2 and grad(dx=P[5] + 2) == -5 and grad(gz=P[6] + 1) == -5 and grad(gv=P[6] + 2) == -5
    for kw in (dict(dx=P[1]), dict(dx=P[0] + 64), dict(dx=P[0], ds=17), dict(dx=P[2]), dict(gv=P[5]), dict(dx=P[3] + 252)):
        assert grad(**kw) == -8, kw


def test_scratch_memory(lib):
    f = lib.rtopk_balance_workspace_bytes
    assert f(1 << 20, 64, BF16, 2, 1) > 0 and f(16, 64, BF16, 2, 1) == 0 and f(1 << 20, 64, BF16, 2, 1 << 20) == 0
    for bad in ((0, 64, F32, 2, 1), (10, 0, F32, 2, 1), (10, 1025, F32, 2, 1), (10, 64, 5, 2, 1), (10, 64, F32, 0, 1), (10, 64, F32, 65, 1), (10, 64, F32, 2, 3), (10, 64, F32, 2, 0)):
        assert f(*bad) == 0


LAYOUTS = r"""
#include <stdio.h>
#include "rtopk_balance_shape.hpp"
using namespace rtopk;
int main() {
  long bad = 0, all = 0;
  const int64_t pers[] = {0, 1, 2, 3, 7, 31, 64, 65, 100, 1000, 4096, 99999, 1 << 20, (int64_t)1 << 30, ((int64_t)1 << 31) - 1};
  const int ks[] = {1, 2, 3, 4, 6, 8, 12, 16, 33, 64, 1024};
  const int64_t counts[] = {1, 2, 3, 8, 100, 1000, 1024, 1025, 65536, 1 << 20};
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int E = 1; E <= kMaxExperts; ++E)
      for (int k : ks) {
        if (k > E) continue;
        for (int grad = 0; grad < 2; ++grad) {
          const RouterLanes r = router_lanes(E, dtype, k, grad);
          const int v = dtype == 0 ? 4 : 8;
          if (r.lanes < 1 || r.lanes > 64 || (r.lanes & (r.lanes - 1)) || r.lanes * r.loads * v < E) ++bad;
          if (E % v == 0 ? (r.lanes * r.loads - r.lanes) * v >= E && r.loads > 1 && r.lanes > 1 && r.lanes * v >= E : false) ++bad;  // no load that all lanes lack
          bool compiled = false;
#define X(n, l) compiled |= r.lanes == n && r.loads == l && is_router_of(dtype, l);
          RTOPK_ROUTER_LIST(X)
#undef X
          if (!compiled) ++bad;
          for (int64_t per : pers)
            for (int64_t groups : counts)
              for (int spread = 0; spread < 2; ++spread) {
                const BalanceLayout l = balance_layout(groups, per, r, spread);
                ++all;
                // every token in one workgroup, none empty unless the group is
                if (l.per_group < 1 || l.rows * l.per_group < per || (l.per_group > 1 && l.rows * (l.per_group - 1) >= per)) ++bad;
                if (!spread && l.per_group != 1) ++bad;
                if (groups * l.per_group > ((int64_t)1 << 23)) ++bad;  // 2^31 threads
              }
        }
      }
  printf("%ld %ld\n", bad, all);
  return bad != 0;
}
"""


def test_layouts(tmp_path):
    src = tmp_path / "layouts.cpp"
    src.write_text(LAYOUTS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(src), "-o", str(tmp_path / "layouts")])
    out = subprocess.run([str(tmp_path / "layouts")], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


def test_definitions_against_differences():
    rng = np.random.default_rng(3)
    N, E, k, groups, h = 12, 5, 2, 2, 1e-6
    x = rng.normal(size=(N, E))
    cols = np.argsort(-x, axis=1)[:, :k]
    cols[4] = -1
    gl, gz, gv = rng.normal(size=groups), rng.normal(size=groups), rng.normal(size=(N, k))
    _, _, _, counts, rows = definition.loss(x, cols, groups)
    assert rows.tolist() == [5, 6] and counts.sum(1).tolist() == [10, 12]

    def value(y):
        loss, z, _, _, _ = definition.loss(y, cols, groups)
        real = cols >= 0
        return (loss * gl).sum() + (z * gz).sum() + (gv * np.take_along_axis(y, np.where(real, cols, 0), 1) * real).sum()

    got = definition.gradient(x, cols, counts, rows, gl, gz, gv)
    for n in range(N):
        for e in range(E):
            y, w = x.copy(), x.copy()
            y[n, e] += h
            w[n, e] -= h
            assert abs((value(y) - value(w)) / (2 * h) - got[n, e]) < 1e-8


def test_even_picks_have_a_loss_of_one():
    x = np.zeros((8, 4))
    cols = np.arange(16).reshape(8, 2) % 4
    loss, z, probs, counts, rows = definition.loss(x, cols)
    assert abs(loss[0] - 1) < 1e-15 and abs(z[0] - np.log(4) ** 2) < 1e-15 and counts.tolist() == [[4, 4, 4, 4]] and rows.tolist() == [8]
