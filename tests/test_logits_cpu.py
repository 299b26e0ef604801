"""Operators on rows of logits without a GPU: arguments refused on the host, the layout of every call, and the definitions themselves
(oracle/logits.py) against differences."""
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT
from oracle import logits as definition


@pytest.fixture(scope="module")
def lib():
    import paper_2409_00822_amd as R

    if not os.path.exists(R.lib_path()):
        from paper_2409_00822_amd import build

        build.build()
    return R.load_library()


P = [1 << 30, 1 << 32, 1 << 34, 1 << 36, 1 << 38, 1 << 40, 1 << 42, 1 << 44]  # far apart, aligned, never dereferenced
F32, F16, BF16 = 0, 1, 2


def test_token_logprobs_refusals(lib):
    def call(x=P[0], dtype=F32, N=4, M=1000, stride=1000, tokens=P[1], token_bytes=8, G=1, k=5, T=1.0, lp=P[2], h=P[3], lse=P[4], tl=P[5], tc=P[6], ws=None, n=0):
        return lib.rtopk_token_logprobs(x, dtype, N, M, stride, tokens, token_bytes, G, k, T, lp, h, lse, tl, tc, ws, n, None)

    assert call(N=0) == 0 and call(N=0, x=None, tokens=None, lp=None) == 0
    for kw in (dict(x=None), dict(tokens=None), dict(lp=None), dict(tl=None), dict(tc=None)):
        assert call(**kw) == -1, kw
    for kw in (dict(N=-1), dict(M=0), dict(stride=999), dict(G=-1), dict(G=1025), dict(k=-1), dict(k=129), dict(M=4, stride=4), dict(n=-1), dict(stride=2**62),
               dict(N=2**40, stride=2**30)):
        assert call(**kw) == -2, kw
    assert call(M=(1 << 24) + 1, stride=1 << 25) == -4
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-42, 3.4e38 * 10):
        assert call(T=T) == -9, T
    for kw in (dict(dtype=3), dict(dtype=-1), dict(token_bytes=2), dict(token_bytes=16)):
        assert call(**kw) == -10, kw
    for kw in (dict(x=P[0] + 2), dict(tokens=P[1] + 4), dict(lp=P[2] + 1), dict(h=P[3] + 2), dict(lse=P[4] + 3), dict(tl=P[5] + 2), dict(tc=P[6] + 1), dict(dtype=F16, x=P[0] + 1),
               dict(ws=P[7] + 8, n=100)):
        assert call(**kw) == -5, kw
    for kw in (dict(lp=P[0]), dict(lp=P[0] + 4 * 3999), dict(h=P[4]), dict(tl=P[6] - 76), dict(tc=P[1] + 28), dict(ws=P[0] + 1024, n=100), dict(lse=P[7], ws=P[7], n=16)):
        assert call(**kw) == -8, kw
    assert lib.rtopk_status_string(-9) != lib.rtopk_status_string(-10) and lib.rtopk_status_string(-10) != b"unknown status"


def test_gradient_refusals(lib):
    def tokens(g=P[0], gh=None, x=P[1], dtype=BF16, N=4, M=1000, stride=1000, t=P[2], token_bytes=4, G=2, lse=P[3], h=None, T=1.0, dx=P[4], ds=1000):
        return lib.rtopk_token_logprobs_backward(g, gh, x, dtype, N, M, stride, t, token_bytes, G, lse, h, T, dx, ds, None)

    def distill(g=P[0], x=P[1], dtype=BF16, N=4, M=1000, stride=1000, tv=P[2], td=F32, tc=P[3], k=8, lp=0, lse=P[4], T=1.0, dx=P[5], ds=1000):
        return lib.rtopk_distill_backward(g, x, dtype, N, M, stride, tv, td, tc, k, lp, lse, T, dx, ds, None)

    def both(g=P[0], x=P[1], dtype=BF16, N=4, M=1000, stride=1000, tv=P[2], td=F32, tc=P[3], k=8, lp=0, T=1.0, loss=P[4], dx=P[5], ds=1000, ws=None, n=0):
        return lib.rtopk_distill_with_grad(g, x, dtype, N, M, stride, tv, td, tc, k, lp, T, loss, dx, ds, ws, n, None)

    for f in (tokens, distill, both):
        assert f(N=0) == 0
        for kw in (dict(g=None), dict(x=None), dict(dx=None)):
            assert f(**kw) == -1, (f, kw)
        for kw in (dict(N=-2), dict(M=0), dict(stride=10), dict(ds=999)):
            assert f(**kw) == -2, (f, kw)
        assert f(T=-0.5) == -9 and f(dtype=7) == -10 and f(x=P[1] + 1) == -5 and f(dx=P[5] + 1) == -5 and f(g=P[0] + 2) == -5
        # the gradient may take its logits' place, but overlap them in no other way
        for kw in (dict(dx=P[1] + 2), dict(dx=P[1], ds=1001), dict(dx=P[1] + 7998), dict(dx=P[0])):
            assert f(**kw) == -8, (f, kw)
    assert tokens(gh=P[5]) == -1 and tokens(lse=None) == -1 and tokens(t=None) == -1 and tokens(G=1025) == -2 and tokens(token_bytes=3) == -10
    assert distill(lse=None) == -1 and both(loss=None) == -1 and both(loss=P[0]) == -8
    for f in (distill, both):
        assert f(k=0) == -2 and f(k=1025) == -2 and f(lp=2) == -2 and f(td=4) == -10 and f(tv=None) == -1 and f(tc=None) == -1 and f(tc=P[3] + 2) == -5
        assert f(td=F16, tv=P[2] + 1) == -5


def test_distill_refusals(lib):
    def call(x=P[0], dtype=F16, N=4, M=1000, stride=1000, tv=P[1], td=F32, tc=P[2], k=8, lp=0, T=1.0, loss=P[3], lse=P[4], ws=None, n=0):
        return lib.rtopk_distill(x, dtype, N, M, stride, tv, td, tc, k, lp, T, loss, lse, ws, n, None)

    assert call(N=0) == 0 and call(loss=None) == -1 and call(tv=None) == -1 and call(k=2000) == -2 and call(lp=-1) == -2 and call(T=0.0) == -9
    assert call(td=5) == -10 and call(lse=P[3]) == -8 and call(loss=P[0] + 4) == -8 and call(loss=P[3] + 2) == -5 and call(n=-5) == -2


def test_scratch_memory(lib):
    f = lib.rtopk_logits_workspace_bytes
    assert f(1, 131072, BF16, 20) > 0 and f(4096, 131072, BF16, 20) == 0 and f(0, 100, F32, 0) == 0 and f(1, 0, F32, 0) == 0
    assert f(1, 131072, 3, 0) == 0 and f(1, 131072, F32, 129) == 0 and f(1, 5, F32, 6) == 0 and f(1, (1 << 24) + 1, F32, 0) == 0


LAYOUTS = r"""
#include <stdio.h>
#include "rtopk_logits_shape.hpp"
using namespace rtopk;
int main() {
  long bad = 0, split = 0, all = 0;
  const int64_t counts[] = {1, 2, 3, 16, 31, 64, 100, 255, 256, 257, 511, 512, 513, 1000, 4096, 100000, (int64_t)1 << 31};
  const int ks[] = {0, 1, 5, 20, 32, 33, 64, 100, 128};
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int64_t M = 1; M <= kMaxLogitsM; M += M < 20000 ? 7 : M / 97)
      for (int64_t N : counts) {
        for (int k : ks) {
          if (k > M) continue;
          const LogitsLayout l = logits_layout(N, (int)M, dtype, k);
          ++all;
          split += l.segments > 1;
          // every column in one segment, none empty
          if (l.segments < 1 || l.segments > kMaxLogitsSegments || (int64_t)l.segments * l.cols < M || (int64_t)(l.segments - 1) * l.cols >= M) ++bad;
          if (l.segments > 1 && (l.cols % logits_width(dtype) != 0 || l.waves != 4 || l.segments * (k > 0 ? k : 1) > kMaxMergeKeys)) ++bad;
          if (l.waves != 1 && l.waves != 4 && l.waves != 8 && l.waves != 16) ++bad;
          // the alternatives' search: threads that hold no column, or at least k, or a row that is listed whole
          if (l.waves == 1 && k > 32) ++bad;
          if (logits_workspace(N, l, k) != (l.segments > 1 ? N * l.segments * (16 + 8 * (int64_t)k) : 0)) ++bad;
        }
        for (int place = 0; place < 2; ++place) {
          const LogitsLayout g = logits_grad_layout(N, (int)M, dtype, place);
          if (g.segments < 1 || (int64_t)g.segments * g.cols < M || (int64_t)(g.segments - 1) * g.cols >= M) ++bad;
          if (g.segments > 1 && g.cols % logits_width(dtype) != 0) ++bad;
          if (place && g.segments != 1) ++bad;
          if (g.segments > (1 << 21)) ++bad;  // a row's workgroups fit a launch
        }
      }
  printf("%ld %ld %ld\n", bad, split, all);
  return 0;
}
"""


def test_layout_of_every_call(tmp_path):
    src = tmp_path / "layouts.cpp"
    src.write_text(LAYOUTS)
    exe = tmp_path / "layouts"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    bad, split, total = map(int, subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    assert bad == 0 and 0 < split < total


def test_host_tensors_are_refused():
    import torch

    import paper_2409_00822_amd as R

    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    v, c, w = torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4)
    for call in (lambda: R.rtopk_token_logprobs(x, t), lambda: R.rtopk_token_logprobs_backward(w, x, t, w), lambda: R.rtopk_distill(x, v, c),
                 lambda: R.rtopk_distill_backward(w, x, v, c, w), lambda: R.rtopk_distill_with_grad(w, x, v, c)):
        with pytest.raises(ValueError):
            call()


def test_definitions_against_differences():
    """Central differences with h = 1e-5: off by h^2 / 6 of third derivatives below 50, and by 2^-52 |value| / h."""
    rng = np.random.default_rng(1)
    N, M, T, h = 3, 9, 0.7, 1e-5
    x = rng.normal(size=(N, M)) * 2
    x[1, 4] = -np.inf
    tokens, g, gh = np.array([[0, 0], [8, -1], [9, 3]]), rng.normal(size=(N, 2)), rng.normal(size=N)
    vals, cols, w = rng.normal(size=(N, 4)), np.array([[0, 3, 3, 8], [1, -1, 2, 9], [-1, -1, -1, -1]]), rng.normal(size=N)

    def policy(v):
        return (definition.token_logprobs(v, tokens, T) * g).sum() + (definition.entropy(definition.log_softmax(v, T)[0]) * gh).sum()

    cases = [(policy, definition.token_gradient(x, tokens, g, gh, T))]
    for lp in (False, True):
        cases.append((lambda v, lp=lp: (definition.distill(v, vals, cols, T, lp) * w).sum(), definition.distill_gradient(x, vals, cols, w, T, lp)))
    for f, d in cases:
        for n in range(N):
            for v in range(M):
                if x[n, v] == -np.inf:
                    assert d[n, v] == 0
                    continue
                up, down = x.copy(), x.copy()
                up[n, v] += h
                down[n, v] -= h
                assert abs(d[n, v] - (f(up) - f(down)) / (2 * h)) < 50 * h * h / 6 + 2.0**-52 * 100 / h


def test_definitions_on_rows_without_columns_left():
    x = np.full((2, 5), -np.inf)
    x[1, 2] = 1.0
    logq, lse = definition.log_softmax(x)
    assert lse[0] == -np.inf and lse[1] == 1.0 and (logq[0] == -np.inf).all() and logq[1, 2] == 0
    assert (definition.entropy(logq) == 0).all()
    assert (definition.token_gradient(x, np.zeros((2, 1), dtype=np.int64), np.ones((2, 1)))[0] == 0).all()
    assert list(definition.top(x, 3)[1]) == [2, 0, 1]
