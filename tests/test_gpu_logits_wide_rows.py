"""Rows of more than 128 KiB, each by one workgroup: held on chip up to 256 KiB, read twice beyond.  Few of them are spread over workgroups where there is scratch
memory, so these calls are made without (tolerances as derived in test_gpu_logits.py).  Which kernel takes a row: test_logits_layouts_cpu.py."""
import types

import numpy as np
import pytest
from test_gpu_logits import MASKS, _gpu, check_distill, check_forward, rows, some_tokens, teacher_list, torch, whole
from test_gpu_logits_in_place import whole_distill, whole_distill_with_grad

pytestmark = pytest.mark.gpu


def without_scratch(R):
    """The public entry points with the forward calls made without scratch memory."""
    return types.SimpleNamespace(rtopk_distill=lambda x, vals, cols, T, log_probs: whole_distill(R, x, vals, cols, T, log_probs),
                                 rtopk_distill_backward=R.rtopk_distill_backward,
                                 rtopk_distill_with_grad=lambda w, x, vals, cols, T, log_probs, grad_logits: whole_distill_with_grad(R, w, x, vals, cols, T, log_probs, grad_logits))


# columns (fp32; twice that in 16 bits) on both sides of what each kernel holds
EDGES = [32768, 49152, 65536]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", EDGES)
@pytest.mark.parametrize("more,shift,pad", [(0, 0, 0), (0, 1, 2), (1, 0, 0), (3, 3, 1), (-1, 1, 0), (-5, 2, 3)])
def test_every_kernel_that_holds_a_row(dtype, M, more, shift, pad):
    R = without_scratch(_gpu())
    M = M * (1 if dtype == "f32" else 2) + more
    x, xh = rows(3, M, dtype, seed=M + shift, pad=pad, shift=shift)
    check_distill(R, x, xh, teacher_list(3, M, 40, M, sort=more >= 0), 0.7 if shift else 1.0, False, dtype, 3, in_place=shift % 2 == 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", ["a tail of -inf", "few columns left", "none left", "one left", "the type's lowest value", "all the type's lowest value", "all equal", "one far above"])
def test_under_masks(mask, dtype):
    R = without_scratch(_gpu())
    for M in (40001, 60000, 65537):
        M *= 1 if dtype == "f32" else 2
        for in_place in (False, True):
            x, xh = rows(3, M, dtype, seed=M, mask=MASKS[mask], shift=1)
            check_distill(R, x, xh, teacher_list(3, M, 30, M), 1.0, False, dtype, 3, in_place=in_place)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("sort", [True, False])
def test_the_longest_list(dtype, sort):
    """1024 entries beside the rows in LDS; columns that come twice."""
    R = _gpu()
    for M in (49000, 65530, 65541, 70000):
        M *= 1 if dtype == "f32" else 2
        x, xh = rows(3, M, dtype, seed=M)
        vals, cols, vh, ch = teacher_list(3, M, 1024, M, sort=sort)
        cols[1, ::2] = cols[1, 1::2]
        lists = (vals, cols, vh, cols.cpu().numpy().astype(np.int64))
        check_distill(without_scratch(R), x, xh, lists, 1.0, False, dtype, 3)
        check_distill(R, x, xh, lists, 1.0, False, dtype, 3, in_place=True)


@pytest.mark.parametrize("dtype,M", [("f32", 49152), ("f32", 49157), ("f32", 65536), ("f32", 65541), ("f16", 98301), ("bf16", 98304), ("bf16", 131072), ("bf16", 131081)])
def test_rows_enough_for_a_workgroup_each(dtype, M):
    """The public call: as many rows as are not spread."""
    R = _gpu()
    N = 97
    x, xh = rows(N, M, dtype, seed=M, pad=3)
    vals, cols, vh, ch = teacher_list(N, M, 40, M, sort=False)
    w = torch.randn((N,), generator=torch.Generator().manual_seed(M)).cuda()
    w[5] = w[70] = 0
    n = [0, 4, 5, 70, 96]
    loss, dx = R.rtopk_distill_with_grad(w, x, vals, cols)
    kept = x.clone()
    loss2, dx2 = R.rtopk_distill_with_grad(w, x, vals, cols, grad_logits=x)
    assert torch.equal(loss, loss2) and torch.equal(dx, dx2)
    apart = R.rtopk_distill(kept, vals, cols)
    some = types.SimpleNamespace(rtopk_distill=lambda *a, **b: [o[n] for o in apart], rtopk_distill_backward=R.rtopk_distill_backward,
                                 rtopk_distill_with_grad=lambda *a, **b: (loss[n], dx[n]))
    check_distill(some, kept[n], xh[n], (vals[n].contiguous(), cols[n].contiguous(), vh[n], ch[n]), 1.0, False, dtype, 3, weights=w[n].contiguous())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_weight_of_zero_and_a_row_of_nan(dtype):
    """Rows with entries and weight 0 have a loss and no gradient; a row of NaN without entries has neither, one with entries spoils itself only."""
    R = _gpu()
    for M in (50000, 65541):
        M *= 1 if dtype == "f32" else 2
        x, xh = rows(4, M, dtype, seed=M, mask=lambda x, g: x[1:3].fill_(float("nan")))
        vals, cols, vh, ch = teacher_list(4, M, 9, M, spoil=False)
        cols[1] = -1
        w = torch.tensor([0.0, 1.0, 1.0, 2.0], device="cuda")
        for call in (lambda: whole_distill_with_grad(R, w, x, vals, cols), lambda: R.rtopk_distill_with_grad(w, x, vals, cols)):
            loss, dx = call()
            assert loss[1] == 0 and (dx[:2] == 0).all() and torch.isnan(loss[2]) and torch.isnan(dx[2].float()).any()
            assert torch.isfinite(loss[[0, 3]]).all() and torch.isfinite(dx[3].float()).all() and (dx[3] != 0).any()


# ---- alternatives ----

@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("k", [1, 31, 32, 33, 34, 128])
@pytest.mark.parametrize("N", [2, 95, 96])
def test_lines_of_the_spread_rows(dtype, N, k):
    """Up to 32 alternatives and 95 rows a row of more than 128 KiB is spread; with and without scratch memory."""
    R = _gpu()
    for M in (32768, 32769) if dtype == "f32" else (65536, 65537):
        x, xh = rows(N, M, dtype, seed=M, pad=1)
        t = some_tokens(N, M, 1, k)
        n = sorted({0, 1, N // 2, N - 1})
        for got in (R.rtopk_token_logprobs(x, t, k), whole(R, x, t, k)):
            check_forward(R, x[n], xh[n], t[n], k, got=[g[n] for g in got])


@pytest.mark.parametrize("dtype,N,M,k", [("f32", 3, 262144, 20), ("f32", 3, 262147, 32), ("bf16", 2, 524288, 17), ("f16", 1, 1 << 20, 9), ("bf16", 4, 300001, 32)])
@pytest.mark.parametrize("mask", ["all equal", "four levels", "ascending", "descending", "a plateau at the end", "zeros of both signs", "few columns left", "one left", "none left"])
def test_more_alternatives_of_segments_than_are_merged_at_once(mask, dtype, N, M, k):
    """Segments times alternatives above 1024, and all of them at or above the floor where logits are equal."""
    R = _gpu()
    x, xh = rows(N, M, dtype, seed=M, mask=MASKS[mask])
    t = some_tokens(N, M, 1, k)
    check_forward(R, x, xh, t, k)
    check_forward(R, x, xh, t, k, got=whole(R, x, t, k))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [256, 257, 512, 513])
@pytest.mark.parametrize("k", [0, 20, 33])
def test_lines_between_sixteen_eight_and_four_wavefronts(dtype, N, k):
    R = _gpu()
    for M in (2049, 9001):
        x, xh = rows(N, M, dtype, seed=N + M, shift=1)
        t = some_tokens(N, M, 1, k)
        got = R.rtopk_token_logprobs(x, t, k)
        for n in (slice(0, 5), slice(N - 5, N)):
            check_forward(R, x[n], xh[n], t[n], k, got=[g[n] for g in got])
        lists = teacher_list(N, M, 20, M)
        n = slice(0, 5)
        apart = R.rtopk_distill(x, *lists[:2])
        both = R.rtopk_distill_with_grad(torch.ones(N, device="cuda"), x, *lists[:2])
        some = types.SimpleNamespace(rtopk_distill=lambda *a, **b: [o[n] for o in apart], rtopk_distill_backward=R.rtopk_distill_backward,
                                     rtopk_distill_with_grad=lambda *a, **b: [o[n] for o in both])
        check_distill(some, x[n], xh[n], [v[n] for v in lists], 1.0, False, dtype, 3, weights=torch.ones(5, device="cuda"))
