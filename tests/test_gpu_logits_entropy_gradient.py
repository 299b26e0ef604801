"""Gradient of the entropy where grad_entropy / temperature is so large that its product with ln q leaves fp32: a column without probability has gradient 0,
and one with little keeps its value."""
import numpy as np
import pytest
from test_gpu_logits import HALF_ULP, MASKS, TYPES, U, _gpu, near, rows, some_tokens, tol_q, torch, wide

from oracle import logits as definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mask", ["a tail of -inf", "few columns left", "one left", "none left", "the type's lowest value"])
@pytest.mark.parametrize("T,g", [(1e-9, 1.0), (1e-20, -3.0), (1e-30, 1.0), (1e-36, 1.0), (1.0, 1e30), (1.0, 1e37)])
def test_columns_without_probability(mask, T, g):
    """Logits are whole numbers, so that at the low temperatures q is 1 / n at the n largest and 0 elsewhere: ln q + H is 0 and the gradient of each is rounding only
    (of H, ln S and exp, 64 units of 2^-24 each, over T)."""
    R = _gpu()
    for N, M in ((3, 1001), (3, 40001), (600, 2001)):
        x, _ = rows(N, M, "f32", seed=M, mask=MASKS[mask])
        x.copy_(torch.round(x))
        xh = wide(x)
        t = torch.zeros((N, 0), dtype=torch.int64, device="cuda")
        ge = torch.full((N,), g, device="cuda")
        _, h, lse = R.rtopk_token_logprobs(x, t, 0, T)
        dx = R.rtopk_token_logprobs_backward(torch.empty((N, 0), device="cuda"), x, t, lse, T, grad_entropy=ge, entropy=h)
        logq, lse_h = definition.log_softmax(xh, T)
        q = np.exp(logq)
        with np.errstate(over="ignore"):
            want = definition.token_gradient(xh, np.empty((N, 0), dtype=np.int64), np.empty((N, 0)), np.full(N, g), T)
        size = q * (np.abs(np.where(q == 0, 0.0, logq)) + definition.entropy(logq)[:, None] + 1)
        tol = abs(g) / T * (tol_q(xh, T, lse_h) * size + 256 * U * q) + U * 1.01 * np.abs(want) + 2.0**-126
        got = wide(dx)
        assert np.isfinite(got).all() and (got[q == 0] == 0).all()
        near(got, want, tol, "gradient")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_little_probability_times_a_large_factor(dtype):
    """q = e^-60, grad_entropy / T = 1e38: the product is finite, ln q + H times the factor alone is not."""
    R = _gpu()
    N, M = 3, 900
    x, _ = rows(N, M, dtype, seed=1, mask=lambda x, g: (x.fill_(-60.0), x[:, 7].fill_(0.0), x[:, 100:].fill_(float("-inf"))))
    xh = wide(x)
    t = torch.zeros((N, 0), dtype=torch.int64, device="cuda")
    scale = {"f32": 1e38, "bf16": 1e38, "f16": 1e29}[dtype]
    _, h, lse = R.rtopk_token_logprobs(x, t, 0)
    # the entropy is given: nought but for 99 e^-60 (60 + 1), so that the large column's own gradient is 0 too
    dx = wide(R.rtopk_token_logprobs_backward(torch.empty((N, 0), device="cuda"), x, t, lse, grad_entropy=torch.full((N,), scale, device="cuda"), entropy=torch.zeros_like(h)))
    q = np.exp(-60.0)
    want = np.zeros((N, M))
    want[:, :100] = scale * q * 60.0
    want[:, 7] = 0.0
    near(dx, want, np.abs(want) * (U * (64 + 4 * 60) + HALF_ULP[dtype] * 1.01), "gradient")
