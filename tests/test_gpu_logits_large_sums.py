"""Gradients where a saved log-sum-exp is so large that a row's sums are taken again: few workgroups of a row do it and write several segments each.  A row's gradient
has the same bits as in a call of a few rows, which test_gpu_logits_layouts.py holds against the definitions; here a few rows are held against them too."""
import numpy as np
import pytest
from test_gpu_logits import HALF_ULP, TINY, U, _gpu, near, rows, some_tokens, teacher_list, tol_q, torch, wide

from oracle import logits as definition

pytestmark = pytest.mark.gpu

# rows of 5 to 12 segments in groups of all sizes, the last one a partial one in some; and of four segments or fewer
SHAPES = [("f32", 100, 24001), ("f32", 300, 24003), ("f32", 700, 20500), ("f32", 60, 48000), ("bf16", 150, 49153), ("f16", 90, 98304), ("bf16", 600, 41001), ("bf16", 1100, 20001), ("f32", 2, 1000003)]


@pytest.mark.parametrize("dtype,N,M", SHAPES)
@pytest.mark.parametrize("entropy", [False, True])
def test_gradient_of_log_probabilities(dtype, N, M, entropy):
    R = _gpu()
    T, G = 0.25, 3
    x, xh = rows(N, M, dtype, seed=N, scale=500.0, pad=7, shift=1)
    some = sorted({0, 1, 2 % N, N // 2, N - 1})
    t = some_tokens(N, M, G, N)
    t[0] = torch.tensor([0, M - 1, M // 3])
    t[N // 2] = -1  # left out: zeros, but for the entropy's gradient
    gen = torch.Generator().manual_seed(N)
    g, ge = torch.randn((N, G), generator=gen).cuda(), torch.randn((N,), generator=gen).cuda()
    ge[N // 2] = 0
    _, h, lse = R.rtopk_token_logprobs(x, t, 0, T)
    assert (lse > 1024).all()
    more = lambda rows_: dict(grad_entropy=ge[rows_].contiguous(), entropy=h[rows_].contiguous()) if entropy else {}  # noqa: E731
    dx = R.rtopk_token_logprobs_backward(g, x, t, lse, T, **more(slice(None)))
    assert (dx[N // 2] == 0).all()
    apart = R.rtopk_token_logprobs_backward(g[some].contiguous(), x[some], t[some].contiguous(), lse[some].contiguous(), T, **more(some))
    assert torch.equal(dx[some], apart)
    y = x.clone()
    assert torch.equal(R.rtopk_token_logprobs_backward(g, y, t, lse, T, grad_logits=y, **more(slice(None))), dx)
    xs, th, gh = xh[some], t[some].cpu().numpy(), wide(g[some])
    want = definition.token_gradient(xs, th, gh, wide(ge[some]) if entropy else None, T)
    logq, lse_h = definition.log_softmax(xs, T)
    q, ok = np.exp(logq), (th >= 0) & (th < M)
    size = np.abs(gh * ok).sum(1, keepdims=True) * q
    if entropy:
        size = size + np.abs(wide(ge[some]))[:, None] * q * (np.abs(np.where(q == 0, 0, logq)) + definition.entropy(logq)[:, None] + 1)
    at_tokens = np.zeros_like(want)
    np.add.at(at_tokens, (np.arange(len(some))[:, None], np.where(ok, th, 0)), np.abs(gh * ok))
    near(wide(dx[some]), want, (tol_q(xs, T, lse_h) * size + 8 * U * at_tokens) / T + HALF_ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype], "gradient")


@pytest.mark.parametrize("dtype,N,M", SHAPES)
@pytest.mark.parametrize("k,sort", [(20, True), (300, False)])
def test_gradient_of_distillation(dtype, N, M, k, sort):
    R = _gpu()
    T = 0.25
    x, xh = rows(N, M, dtype, seed=N, scale=500.0, pad=7, shift=1)
    vals, cols, vh, ch = teacher_list(N, M, k, N, sort=sort)
    w = torch.randn((N,), generator=torch.Generator().manual_seed(N)).cuda()
    w[N // 2] = 0
    _, lse = R.rtopk_distill(x, vals, cols, T)
    assert (lse > 1024).all()
    dx = R.rtopk_distill_backward(w, x, vals, cols, lse, T)
    some = sorted({0, 1, 2 % N, N // 2, N - 1})
    apart = R.rtopk_distill_backward(w[some].contiguous(), x[some], vals[some].contiguous(), cols[some].contiguous(), lse[some].contiguous(), T)
    assert torch.equal(dx[some], apart) and (dx[N // 2] == 0).all()
    y = x.clone()
    assert torch.equal(R.rtopk_distill_backward(w, y, vals, cols, lse, T, grad_logits=y), dx)
    xs, wh = xh[some], wide(w[some])
    want = definition.distill_gradient(xs, vh[some], ch[some], wh, T)
    logq, lse_h = definition.log_softmax(xs, T)
    p, lp, _ = definition.teacher(vh[some], ch[some], M, T)
    # ln p as in test_gpu_logits.py
    t_lp = U * (8 * np.abs(np.where(np.isfinite(vh[some]), vh[some], 0)).max(axis=1, keepdims=True) / T + 2 * np.abs(lp) + 64)
    at_list = np.zeros_like(want)
    np.add.at(at_list, (np.arange(len(some))[:, None], np.where((ch[some] >= 0) & (ch[some] < M), ch[some], 0)), p * (t_lp + 8 * U))
    tol = np.abs(wh)[:, None] / T * (tol_q(xs, T, lse_h) * np.exp(logq) * p.sum(1, keepdims=True) + np.exp(logq) * (p * t_lp).sum(1, keepdims=True) + at_list)
    near(wide(dx[some]), want, tol + HALF_ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype], "gradient")
