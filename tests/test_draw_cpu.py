"""Drawn tokens and verified drafts without a GPU: arguments refused on the host, and the definitions themselves (oracle/draw.py): tokens that come out of
verified drafts are distributed as the target's."""
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT
from oracle import draw as definition


@pytest.fixture(scope="module")
def lib():
    import paper_2409_00822_amd as R

    if not os.path.exists(R.lib_path()):
        from paper_2409_00822_amd import build

        build.build()
    return R.load_library()


P = [1 << 30, 1 << 32, 1 << 34, 1 << 36, 1 << 38, 1 << 40, 1 << 42, 1 << 44]  # far apart, aligned, never dereferenced
F32, F16, BF16 = 0, 1, 2


def test_sample_refusals(lib):
    def call(x=P[0], dtype=F32, N=4, M=1000, stride=1000, u=P[1], temps=None, T=1.0, out=P[2], token_bytes=8, ws=None, n=0):
        return lib.rtopk_sample_tokens(x, dtype, N, M, stride, u, temps, T, out, token_bytes, ws, n, None)

    assert call(N=0) == 0 and call(N=0, x=None, u=None, out=None) == 0
    for kw in (dict(x=None), dict(u=None), dict(out=None), dict(u=None, temps=P[3], T=0.0)):
        assert call(**kw) == -1, kw
    for kw in (dict(N=-1), dict(M=0), dict(stride=999), dict(n=-1), dict(stride=2**62), dict(N=2**40, stride=2**30), dict(N=2**62, stride=1000)):
        assert call(**kw) == -2, kw
    assert call(M=(1 << 24) + 1, stride=1 << 25) == -4
    for T in (-0.5, float("nan"), float("inf"), 1e-320):
        assert call(T=T) == -9, T
    for kw in (dict(dtype=3), dict(dtype=-1), dict(token_bytes=2), dict(token_bytes=0)):
        assert call(**kw) == -10, kw
    for kw in (dict(x=P[0] + 2), dict(u=P[1] + 2), dict(out=P[2] + 4), dict(temps=P[3] + 1), dict(dtype=F16, x=P[0] + 1), dict(ws=P[7] + 8, n=64)):
        assert call(**kw) == -5, kw
    for kw in (dict(out=P[0]), dict(out=P[0] + 8 * 1999), dict(out=P[1] + 8), dict(out=P[3], temps=P[3]), dict(ws=P[0], n=64), dict(ws=P[2] + 16, n=64)):
        assert call(**kw) == -8, kw


def test_verify_refusals(lib):
    def call(x=P[0], q=P[1], dtype=BF16, B=4, G=3, M=1000, xs=4000, xp=1000, qs=3000, qp=1000, d=P[2], token_bytes=8, u=P[3], temps=None, T=1.0, out=P[4], acc=P[5], ws=None, n=0):
        return lib.rtopk_verify_drafts(x, q, dtype, B, G, M, xs, xp, qs, qp, d, token_bytes, u, temps, T, out, acc, ws, n, None)

    assert call(B=0) == 0
    for kw in (dict(x=None), dict(d=None), dict(u=None), dict(out=None)):
        assert call(**kw) == -1, kw
    for kw in (dict(B=-1), dict(G=-1), dict(G=129), dict(M=0), dict(xs=999), dict(xp=999), dict(qs=10), dict(qp=999), dict(xp=2**61), dict(qs=2**61), dict(n=-1), dict(B=2**59)):
        assert call(**kw) == -2, kw
    assert call(M=(1 << 24) + 1, xs=1 << 30, xp=1 << 25, qs=1 << 30, qp=1 << 25) == -4 and call(T=-1.0) == -9 and call(token_bytes=3) == -10 and call(dtype=9) == -10
    for kw in (dict(x=P[0] + 1), dict(q=P[1] + 1), dict(d=P[2] + 4), dict(u=P[3] + 2), dict(out=P[4] + 4), dict(acc=P[5] + 2), dict(ws=P[6] + 4, n=64)):
        assert call(**kw) == -5, kw
    for kw in (dict(out=P[0] + 8), dict(out=P[1] + 8 * 2999), dict(out=P[2]), dict(acc=P[3] + 60), dict(acc=P[4] + 124), dict(ws=P[1], n=64)):
        assert call(**kw) == -8, kw
    # what a call does not look at: draft strides without draft logits, draft logits at a temperature of 0, random numbers there
    assert call(q=None, qs=0, qp=0, x=None) == -1 and call(T=0.0, qs=0, qp=0, out=None) == -1 and call(T=0.0, u=None, out=None) == -1


def test_scratch_memory(lib):
    f = lib.rtopk_verify_workspace_bytes
    for bad in ((0, 0, 100, F32, 0), (1, -1, 100, F32, 0), (1, 129, 100, F32, 0), (1, 1, 0, F32, 0), (1, 1, (1 << 24) + 1, F32, 0), (1, 1, 100, 3, 0), (1, 1, 100, F32, 2)):
        assert f(*bad) == 0
    for good in ((1, 0, 131072, BF16, 0), (4096, 0, 131072, BF16, 0), (64, 7, 131072, F32, 1), (1 << 40, 0, 100, F32, 0)):
        assert f(*good) >= 0


def test_drawn_tokens_have_the_rows_probabilities():
    rng = np.random.default_rng(1)
    x = rng.normal(size=6) * 2
    for T in (0.5, 1.0, 3.0):
        p = definition.distribution(x, T)
        y = np.exp(x / T)
        assert np.allclose(p, y / y.sum(), rtol=1e-14)
        got = np.bincount([definition.sample(x, u, T)[0] for u in (np.arange(20000) + 0.5) / 20000], minlength=6) / 20000
        assert np.abs(got - p).max() < 1e-4
    assert definition.sample(np.array([1.0, 5.0, 5.0]), 0.99, 0.0)[0] == 1


@pytest.mark.parametrize("with_draft", [True, False])
def test_verified_tokens_have_the_targets_distribution(with_draft):
    rng = np.random.default_rng(2)
    M, n = 4, 60
    target, draft = rng.normal(size=(2, M)) * 2, rng.normal(size=(1, M)) * 2
    p, q = definition.distribution(target[0], 1.0), definition.distribution(draft[0], 1.0)
    grid = (np.arange(n) + 0.5) / n
    first = np.zeros(M)
    second = np.zeros((M, M))  # of the bonus token, by the accepted one
    for d in range(M):
        of = q[d] if with_draft else 1.0 / M  # (looked up: any draft leaves the target's distribution)
        for u0 in grid:
            for u1 in grid:
                tokens, accepted, _ = definition.verify(target, [d], [u0, u1], draft if with_draft else None, 1.0)
                first[tokens[0]] += of / n**2
                if accepted:
                    assert tokens[0] == d
                    second[d, tokens[1]] += of / n**2
    assert np.abs(first - p).max() < 3 / n
    bonus = definition.distribution(target[1], 1.0)
    rows = second / np.maximum(second.sum(1, keepdims=True), 1e-9)
    assert np.abs(rows[second.sum(1) > 0.05] - bonus).max() < 3 / n


def test_hand_traces():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.125, 0.125, 0.75]]))
    q = np.log(np.array([[0.25, 0.25, 0.5]]))
    # p / q of the drafts: 2, 1, 1/2
    assert definition.verify(x, [0], [0.99, 0.2], q, 1.0)[:2] == ([0, 1], 1)
    assert definition.verify(x, [2], [0.49, 0.3], q, 1.0)[:2] == ([2, 2], 1)
    assert definition.verify(x, [2], [0.51, 0.9], q, 1.0)[:2] == ([0, -1], 0)  # all that p has more of is on column 0
    # a draft that stands for itself
    assert definition.verify(x, [1], [0.24, 0.0], None, 1.0)[:2] == ([1, 0], 1)
    assert definition.verify(x, [1], [0.26, 0.6], None, 1.0)[:2] == ([0, -1], 0)
    assert definition.verify(x, [1], [0.26, 0.7], None, 1.0)[:2] == ([2, -1], 0)
    # the largest logits
    assert definition.verify(x, [0], [0.9, 0.9], q, 0.0)[:2] == ([0, 2], 1)
    assert definition.verify(x, [1], [0.0, 0.9], q, 0.0)[:2] == ([0, -1], 0)
    assert definition.verify(x, [-1], [0.0, 0.6], q, 1.0)[:2] == ([1, -1], 0)


CHUNKS = r"""
#include <stdio.h>
// The columns that the lanes of a wavefront read of a piece (piece_mass): each of the piece once, none beyond it.
int main() {
  long bad = 0;
  for (int V = 4; V <= 8; V += 4)
    for (int cols = 1; cols <= 4096; ++cols) {
      static int seen[4200];
      for (int c = 0; c < 4200; ++c) seen[c] = 0;
      const int full = cols / V, rest = cols % V, U = V == 4 ? 4 : 2;
      for (int lane = 0; lane < 64; ++lane) {
        int i = lane;
        const auto whole = [&](int chunk) { for (int c = 0; c < V; ++c) ++seen[chunk * V + c]; };
        for (; i - lane + U * 64 <= full; i += U * 64)
          for (int u = 0; u < U; ++u) whole(i + u * 64);
        for (; i - lane < full; i += 64)
          if (i < full) whole(i);
        if (lane < rest) ++seen[full * V + lane];
      }
      for (int c = 0; c < 4200; ++c) bad += seen[c] != (c < cols);
    }
  printf("%ld\n", bad);
  return bad != 0;
}
"""


def test_the_lanes_of_a_piece_read_its_columns_and_no_others(tmp_path):
    src = tmp_path / "chunks.cpp"
    src.write_text(CHUNKS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(src), "-o", str(tmp_path / "chunks")])
    out = subprocess.run([str(tmp_path / "chunks")], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


LAYOUTS = r"""
#include <stdio.h>
#include "rtopk_draw_shape.hpp"
using namespace rtopk;
int main() {
  long bad = 0, all = 0, tested = 0, spread = 0;
  const int64_t counts[] = {1, 2, 3, 16, 63, 64, 255, 256, 511, 512, 513, 1000, 1024, 4096, 16384, 16385, 100000, (int64_t)1 << 31};
  const int drafts[] = {0, 1, 2, 3, 7, 64, 128};
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int64_t M = 1; M <= kMaxLogitsM; M += M < 20000 ? 7 : M / 97)
      for (int64_t B : counts)
        for (int G : drafts)
          for (int draft = 0; draft <= (G > 0); ++draft) {
            const DrawLayout l = draw_layout(B, G, (int)M, dtype, draft);
            ++all;
            tested += l.tested;
            spread += l.spread;
            // every column in one piece, none empty, whole loads of a wavefront
            if (l.pieces < 1 || (int64_t)l.pieces * l.cols < M || (int64_t)(l.pieces - 1) * l.cols >= M || l.cols % (64 * logits_width(dtype)) != 0) ++bad;
            if (l.pieces > (l.spread ? 1024 : kMostPieces)) ++bad;
            if (l.waves != 1 && l.waves != 4 && l.waves != 8 && l.waves != 16) ++bad;
            if (l.tested && (!l.spread || G == 0 || M > kMostTested || l.positions < 1 || (l.test_waves != 4 && l.test_waves != 8 && l.test_waves != 16))) ++bad;
            if (l.groups < 1 || (l.spread && l.groups > (l.pieces + kDrawWaves - 1) / kDrawWaves)) ++bad;
            // a sequence's workgroups fit a launch
            if (l.spread && (int64_t)draw_rows(G, draft) * ((l.pieces + kDrawWaves - 1) / kDrawWaves) > (1 << 21)) ++bad;
            const int64_t bytes = draw_workspace(B, G, draft, l);
            if (bytes < 0 || (l.spread ? bytes < 16 * B * l.pieces : bytes != 0)) ++bad;
            const DrawLayout w = draw_layout_whole(B, (int)M, dtype);
            if (w.spread || w.pieces > kMostPieces || (int64_t)w.pieces * w.cols < M) ++bad;
          }
  printf("%ld of %ld, %ld spread, %ld tested\n", bad, all, spread, tested);
  return bad != 0 || tested == 0 || spread == 0;
}
"""


def test_layouts(tmp_path):
    src = tmp_path / "layouts.cpp"
    src.write_text(LAYOUTS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(src), "-o", str(tmp_path / "layouts")])
    out = subprocess.run([str(tmp_path / "layouts")], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
