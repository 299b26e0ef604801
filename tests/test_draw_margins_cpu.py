"""What the fp32 sums may be off by that drafts are tested with, without a GPU: the count of their roundings (test_units) against the same additions, made here in fp32 in the
order of a workgroup's threads, of rows on which roundings add up."""
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT

F = np.float32
U = 2.0**-24
C = F(1.44269504088896340736)

COUNTS = r"""
#include <stdio.h>
#include <stdlib.h>
#include "rtopk_draw_shape.hpp"
using namespace rtopk;
// dtype, M, waves -> units near and far, and the margin of two near rows
int main(int n, char** v) {
  const int dtype = atoi(v[1]), M = atoi(v[2]), waves = atoi(v[3]);
  const long near = test_units(M, dtype, waves, false), far = test_units(M, dtype, waves, true);
  printf("%ld %ld %.17g %d\n", near, far, test_margin(2 * near), test_loads(waves));
}
"""


@pytest.fixture(scope="module")
def counts(tmp_path_factory):
    d = tmp_path_factory.mktemp("counts")
    (d / "counts.cpp").write_text(COUNTS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2409_00822_amd", "csrc"), str(d / "counts.cpp"), "-o", str(d / "counts")])

    def run(dtype, M, waves):
        near, far, margin, loads = subprocess.check_output([str(d / "counts"), str(dtype), str(M), str(waves)], text=True).split()
        return int(near), int(far), float(margin), int(loads)

    return run


def exp2(y, late):
    """A power of two in fp32; late: off by a unit of its last place, upwards or downwards, as the GPU's may be."""
    e = np.exp2(y.astype(np.float64))
    return np.nextafter(e.astype(F), F(late * np.inf)) if late else e.astype(F)


def near_sum(x, threads, loads, width, late):
    """Sum of 2^((x - max) C), threads one behind the other over batches of `loads` loads of `width` columns each; M a multiple of all that."""
    x = x.reshape(-1, loads, threads, width)
    m = np.full(threads, -np.inf, dtype=F)
    s = np.zeros(threads, dtype=F)
    reference = lambda m: np.maximum(m * C, F(-(2.0**20)))

    def rise(m, s, to):
        with np.errstate(invalid="ignore"):
            d = reference(m) - reference(to)
        return s * np.where(d == 0, F(1), exp2(d, late))

    for batch in x:
        to = np.maximum(m, batch.max((0, 2)))
        s, m = rise(m, s, to), to
        r = reference(m)
        a = [np.zeros(threads, dtype=F), np.zeros(threads, dtype=F)]
        for i in range(loads * width):
            y = (batch[i // width, :, i % width].astype(np.float64) * float(C) - r).astype(F)  # (one rounding, but for 2^-53)
            a[i & 1] = a[i & 1] + exp2(y, late)
        s = s + (a[0] + a[1])
    for n in (64, threads // 64):  # a wavefront's lanes, then the wavefronts
        m, s = m.reshape(-1, n), s.reshape(-1, n)
        top = m.max(1, keepdims=True)
        s, m = rise(m, s, top), top[:, 0]
        while s.shape[1] > 1:
            s = s[:, ::2] + s[:, 1::2]
        s = s[:, 0]
    off = F(float(m[0]) * float(C) - float(reference(m)[0]))
    return float(s[0] * exp2(np.array([-off], dtype=F), late)[0])


def far_sum(x, threads, width, late):
    top = x.max()
    x = x.reshape(-1, threads, width)
    s = np.zeros(threads, dtype=F)
    for chunk in x:
        for i in range(width):
            s = s + exp2((chunk[:, i] - top) * C, late)
    while s.size > 1:
        s = s[::2] + s[1::2]
    return float(s[0])


def exact(x):
    x = x.astype(np.float64)
    return float(np.exp(x - x.max()).sum())


def rows(M, threads, loads, width, rng):
    """Rows whose maxima rise all along, by little or by much, in the columns of a batch of the threads' loads at a time."""
    chunk = threads * loads * width
    at = np.arange(M) // chunk
    yield (at * 2.0**-8).astype(F)
    yield (at * 2.0**-5 - 3 * rng.random(M)).astype(F)
    first = np.where(at == 0, 0.0, -30.0)  # all that weighs in the first batch, and a new maximum in each
    first.reshape(-1, loads, threads, width)[:, 0, :, 0] = at[::chunk, None] * 2.0**-12
    yield first.astype(F)
    yield (8 * rng.standard_normal(M)).astype(F)
    yield (1000.0 + 2 * rng.standard_normal(M)).astype(F)


@pytest.mark.parametrize("dtype,M,waves", [(0, 1 << 20, 4), (0, 1 << 17, 4), (0, 1 << 18, 8), (0, 1 << 17, 16), (2, 1 << 18, 4), (2, 1 << 15, 8)])
@pytest.mark.parametrize("late", [0, 1, -1])
def test_sums_are_off_by_no_more_than_is_counted(counts, dtype, M, waves, late):
    near, far, margin, loads = counts(dtype, M, waves)
    width, threads = (4, 8)[dtype != 0], 64 * waves
    assert near < 900 and margin > 2 * near * U
    worst = 0.0
    for x in rows(M, threads, loads, width, np.random.default_rng(1)):
        want = exact(x)
        worst = max(worst, abs(near_sum(x, threads, loads, width, late) - want) / want / U)
    assert worst <= near, (worst, near)
    print(worst, near)


@pytest.mark.parametrize("M,waves", [(1 << 20, 4), (1 << 20, 16), (1 << 17, 8)])
@pytest.mark.parametrize("late", [0, 1, -1])
def test_sums_of_rows_far_from_zero(counts, M, waves, late):
    near, far, _, _ = counts(0, M, waves)
    worst = 0.0
    for k in (1, 6, 11, 20, 37):
        x = (2.0**20 - np.where(np.arange(M) == 5, 0, k) / 8.0).astype(F)
        want = exact(x)
        worst = max(worst, abs(far_sum(x, 64 * waves, 4, late) - want) / want / U)
    assert worst <= far, (worst, far)
    assert M < 1 << 20 or waves > 4 or worst > near / 2  # (more than rows near zero have)
