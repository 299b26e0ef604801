"""Loss and gradient in one call with the gradient in its logits' place: the loss is that of the logits, whatever the rows' weights are (tolerances as
derived in test_gpu_logits.py)."""
import numpy as np
import pytest
from test_gpu_logits import _gpu, near, rows, teacher_list, tol_distill, torch, wide

from oracle import logits as definition

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def whole_distill(R, x, vals, cols, T=1.0, log_probs=False):
    """rtopk_distill without scratch memory: a workgroup for each row."""
    N, M = x.shape
    loss, lse = (torch.full((N,), 7.5, device="cuda") for _ in range(2))
    rc = R.load_library().rtopk_distill(x.data_ptr(), TYPES.index(x.dtype), N, M, x.stride(0), vals.data_ptr(), TYPES.index(vals.dtype), cols.data_ptr(), vals.shape[1], int(log_probs), T,
                                        loss.data_ptr(), lse.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    return loss, lse


def whole_distill_with_grad(R, weights, x, vals, cols, T=1.0, log_probs=False, grad=None):
    """rtopk_distill_with_grad without scratch memory; grad: None for new rows."""
    N, M = x.shape
    loss = torch.full((N,), 7.5, device="cuda")
    if grad is None:
        grad = torch.full((N, M), 7.5, dtype=x.dtype, device="cuda")
    rc = R.load_library().rtopk_distill_with_grad(weights.data_ptr(), x.data_ptr(), TYPES.index(x.dtype), N, M, x.stride(0), vals.data_ptr(), TYPES.index(vals.dtype), cols.data_ptr(),
                                                  vals.shape[1], int(log_probs), T, loss.data_ptr(), grad.data_ptr(), grad.stride(0), None, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    return loss, grad


def check_weights_of_zero(R, N, M, dtype, k, whole):
    """A third of the rows, with entries, has weight 0, as padded positions do; one row has nothing but -inf."""
    x, xh = rows(N, M, dtype, seed=M + k, mask=lambda x, g: x[N // 2].fill_(float("-inf")))
    vals, cols, vh, ch = teacher_list(N, M, k, M, sort=False, spoil=False)
    weights = torch.rand((N,), generator=torch.Generator().manual_seed(k)) + 0.5
    weights[::3] = 0
    weights = weights.cuda()
    call = (lambda grad: whole_distill_with_grad(R, weights, x, vals, cols, grad=grad)) if whole else (lambda grad: R.rtopk_distill_with_grad(weights, x, vals, cols, grad_logits=grad))
    loss, dx = call(None)
    apart, _ = R.rtopk_distill(x, vals, cols)
    kept = x.clone()
    for _ in range(3):
        x.copy_(kept)
        loss2, dx2 = call(x)
        assert torch.equal(loss2, loss) and torch.equal(dx2, dx)
    some = sorted({0, 1, 2, N // 2, N - 2, N - 1} | set(range(0, N, max(1, N // 8))))
    want, tol = definition.distill(xh[some], vh[some], ch[some]), tol_distill(xh[some], vh[some], ch[some], 1.0, False)[0]
    near(wide(loss[some]), want, tol, "loss")
    near(wide(apart[some]), want, tol, "loss by itself")
    assert (dx[::3] == 0).all() and (dx[N // 2] == 0).all()
    rest = [n for n in range(N) if n % 3 and n != N // 2]
    assert (dx[rest] != 0).any(dim=1).all()


@pytest.mark.parametrize("dtype,M", [("f32", 65541), ("f16", 131073), ("bf16", 131081)])
@pytest.mark.parametrize("k", [1, 40, 1024])
def test_rows_too_wide_to_hold(dtype, M, k):
    R = _gpu()
    check_weights_of_zero(R, 97, M, dtype, k, whole=False)
    check_weights_of_zero(R, 3, M, dtype, k, whole=True)


@pytest.mark.parametrize("dtype,N,M", [("f32", 5, 3000), ("bf16", 5, 3001), ("f32", 4, 65541), ("bf16", 4, 131081), ("bf16", 100, 65543), ("f32", 100, 49999)])
def test_every_other_form(dtype, N, M):
    """Held on chip, and few wide rows over several workgroups each."""
    R = _gpu()
    for k in (1, 40, 1024):
        check_weights_of_zero(R, N, M, dtype, k, whole=False)
