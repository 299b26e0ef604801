"""Every layout of the operators on rows of logits at its widest and narrowest rows, aligned and not, against the definitions in 64 bits (tolerances as
derived in test_gpu_logits.py)."""
import numpy as np
import pytest
from test_gpu_logits import MASKS, _gpu, check_distill, check_forward, check_token_gradient, rows, some_tokens, teacher_list, torch, whole

pytestmark = pytest.mark.gpu

# rows held on chip: one column below, at and above what each layout holds (fp32; twice that in 16 bits), and the widest
EDGES = [1024, 4096, 8192, 16384, 32768, 49152, 65536]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", EDGES)
def test_rows_held_on_chip(dtype, M):
    R = _gpu()
    M *= 1 if dtype == "f32" else 2
    for more, N, pad in ((-1, 3, 0), (0, 4, 2), (3, 3, 1)):
        x, xh = rows(N, M + more, dtype, seed=M + more, pad=pad, shift=1)
        check_distill(R, x, xh, teacher_list(N, M + more, 40, M, sort=more == 0), 1.0, False, dtype, 3, in_place=more == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", ["a tail of -inf", "few columns left", "none left", "one left", "the type's lowest value", "all the type's lowest value", "all equal"])
def test_rows_held_on_chip_under_masks(mask, dtype):
    R = _gpu()
    for M in (700, 3000, 20000, 60000) if dtype == "f32" else (1500, 9000, 50001, 131000):
        x, xh = rows(3, M, dtype, seed=M, mask=MASKS[mask])
        check_distill(R, x, xh, teacher_list(3, M, 30, M), 1.0, False, dtype, 3)
        check_distill(R, x, xh, teacher_list(3, M, 30, M), 0.5, False, dtype, 3, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_entries_at_the_ends_of_a_row(dtype):
    """The first and last columns, which may lie in a partial chunk or before the first whole one."""
    R = _gpu()
    for M, shift in ((1000, 0), (1001, 1), (4099, 1), (33001, 1), (70001, 1), (140001, 1)):
        x, xh = rows(4, M, dtype, seed=M, shift=shift, pad=shift)
        cols = np.tile(np.concatenate([np.arange(6), np.arange(M - 9, M)]), (4, 1))
        vals = torch.randn(cols.shape, generator=torch.Generator().manual_seed(1))
        lists = (vals.cuda(), torch.from_numpy(cols).int().cuda(), vals.double().numpy(), cols)
        check_distill(R, x, xh, lists, 1.0, False, dtype, 3, in_place=True)
        tokens = torch.tensor([[0, M - 1], [1, M - 2], [M - 1, M - 1], [0, 0]]).cuda()
        x, xh = rows(4, M, dtype, seed=M, shift=shift, pad=shift)
        check_forward(R, x, xh, tokens, 5)
        check_token_gradient(R, x, xh, tokens, 1.0, True, 3, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,M", [(1, 32768), (95, 33001), (96, 33001), (320, 5001), (321, 5001), (4, 66001), (97, 70001)])
@pytest.mark.parametrize("k", [0, 8, 9, 128])
def test_few_rows(dtype, N, M, k):
    """On both sides of the lines between a workgroup of sixteen or four wavefronts to a row and several workgroups to a row."""
    R = _gpu()
    x, xh = rows(N, M, dtype, seed=N + M)
    n = min(N, 7)
    got = R.rtopk_token_logprobs(x, some_tokens(N, M, 1, k), k)
    check_forward(R, x[:n], xh[:n], some_tokens(N, M, 1, k)[:n], k, got=[g[:n] for g in got])
    check_forward(R, x[-n:], xh[-n:], some_tokens(N, M, 1, k)[-n:], k, got=[g[-n:] for g in got])


@pytest.mark.parametrize("mask", list(MASKS))
@pytest.mark.parametrize("N,M,k", [(3, 70001, 20), (2, 20000, 5), (340, 9000, 33)])
def test_alternatives_under_masks_in_every_layout(mask, N, M, k):
    R = _gpu()
    for dtype in ("f32", "bf16"):
        x, xh = rows(N, M, dtype, seed=N + M, mask=MASKS[mask])
        t = some_tokens(N, M, 1, k)
        n = min(N, 6)
        for got in (R.rtopk_token_logprobs(x, t, k), whole(R, x, t, k)):
            check_forward(R, x[:n], xh[:n], t[:n], k, got=[g[:n] for g in got])


def test_low_temperatures():
    """x / T beyond what a difference of fp32 products holds, up to where 1 / T ends."""
    R = _gpu()
    for T in (1e-3, 1e-20, 1e-36):
        for N, M in ((3, 3000), (3, 70000)):
            x, xh = rows(N, M, "f32", seed=M)
            xh = np.round(xh)  # gaps of 1: what lies below the maximum has no share, whatever the rounding
            x.copy_(torch.from_numpy(xh).float())
            got = R.rtopk_token_logprobs(x, torch.from_numpy(xh.argmax(1)).cuda(), 3, T)
            n_top = (xh == xh.max(axis=1, keepdims=True)).sum(axis=1)
            assert np.allclose(got[0].cpu().numpy(), -np.log(n_top), rtol=0, atol=64 * 2.0**-24 * (1 + np.log(n_top)))
            assert np.allclose(got[1].cpu().numpy(), np.log(n_top), rtol=0, atol=64 * 2.0**-24 * (1 + np.log(n_top)))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_log_sum_exps(dtype):
    """Beyond 1024 a saved log-sum-exp has too few digits: the row's sums are taken again, also where the gradient takes its logits' place."""
    R = _gpu()
    for N, M in ((3, 2001), (3, 40001)):
        x, xh = rows(N, M, dtype, seed=M, scale=500.0)
        check_token_gradient(R, x, xh, some_tokens(N, M, 2, 1), 0.25, True, 3, dtype)
        check_distill(R, x, xh, teacher_list(N, M, 20, 3), 0.25, False, dtype, 3)
        t = some_tokens(N, M, 0, 1)
        _, h, lse = R.rtopk_token_logprobs(x, t, 0, 0.25)
        g = torch.randn((N,), device="cuda")
        want = R.rtopk_token_logprobs_backward(g, x, t, lse, 0.25)
        y = x.clone()
        assert torch.equal(R.rtopk_token_logprobs_backward(g, y, t, lse, 0.25, grad_logits=y), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [-1e4, -1e9, -1e20, -1e30])
@pytest.mark.parametrize("keep", [0.0, 0.002, 0.5])
def test_masks_of_large_negative_values(value, keep, dtype):
    R = _gpu()
    mask = lambda x, g: x.masked_fill_(torch.rand(x.shape, generator=g) >= keep, value)  # noqa: E731
    for N, M in ((3, 1500), (3, 30000), (3, 90000), (330, 2300)):
        x, xh = rows(N, M, dtype, seed=M, mask=mask)
        for k in (0, 20):
            check_forward(R, x, xh, some_tokens(N, M, 1, 1), k)
        check_token_gradient(R, x, xh, some_tokens(N, M, 1, 1), 1.0, True, 3, dtype)
        check_distill(R, x, xh, teacher_list(N, M, 20, 3), 1.0, False, dtype, 3)


def test_a_teacher_of_nan_spoils_its_row_only():
    """Alike in all forms: NaN loss and gradient, and only there."""
    R = _gpu()
    for N, M in ((5, 3000), (5, 70000), (5, 140001), (600, 2500)):
        x, _ = rows(N, M, "f32", seed=1)
        vals, cols, _, _ = teacher_list(N, M, 6, 2, spoil=False)
        vals[1] = float("nan")
        vals[3, 2] = float("nan")
        w = torch.ones(N, device="cuda")
        loss, lse = R.rtopk_distill(x, vals, cols)
        loss2, dx = R.rtopk_distill_with_grad(w, x, vals, cols)
        dx2 = R.rtopk_distill_backward(w, x, vals, cols, lse)
        bad = torch.zeros(N, dtype=torch.bool, device="cuda")
        bad[1] = bad[3] = True
        for o in (loss, loss2, dx.sum(1), dx2.sum(1)):
            assert torch.equal(torch.isnan(o), bad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mask", ["none", "few columns left", "none left", "all equal", "four levels", "ascending", "the largest where a few threads read", "a plateau at the end"])
def test_eight_wavefronts_to_a_row(mask, dtype):
    R = _gpu()
    for N, M, k in ((257, 2300, 128), (400, 9001, 20), (512, 20003, 1)):
        x, xh = rows(N, M, dtype, seed=N + M, mask=MASKS.get(mask))
        t = some_tokens(N, M, 1, k)
        got = R.rtopk_token_logprobs(x, t, k)
        check_forward(R, x[:9], xh[:9], t[:9], k, got=[g[:9] for g in got])
        check_forward(R, x[-9:], xh[-9:], t[-9:], k, got=[g[-9:] for g in got])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mask", ["none", "few columns left", "none left", "all equal", "four levels", "ascending", "the type's lowest value", "a plateau at the end"])
def test_one_wavefront_to_a_row(mask, dtype):
    R = _gpu()
    for N, M, k in ((4096, 2049, 32), (4100, 4999, 20), (4097, 700, 5), (4096, 16384, 1)):
        x, xh = rows(N, M, dtype, seed=N + M, mask=MASKS.get(mask))
        t = some_tokens(N, M, 1, k)
        got = R.rtopk_token_logprobs(x, t, k)
        check_forward(R, x[:9], xh[:9], t[:9], k, got=[g[:9] for g in got])
        check_forward(R, x[-9:], xh[-9:], t[-9:], k, got=[g[-9:] for g in got])
        lists = teacher_list(9, M, 20, 3)
        loss, _ = R.rtopk_distill(x, lists[0].repeat(N // 9 + 1, 1)[:N].contiguous(), lists[1].repeat(N // 9 + 1, 1)[:N].contiguous())
        want, _ = R.rtopk_distill(x[:9], *lists[:2])  # (another layout, checked elsewhere)
        finite = torch.isfinite(want)
        assert torch.equal(finite, torch.isfinite(loss[:9]))
        torch.testing.assert_close(loss[:9][finite], want[finite], rtol=1e-5, atol=1e-5)
