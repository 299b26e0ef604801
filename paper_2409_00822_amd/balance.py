"""A router's balance loss and its gradient, with the names of the C ABI (include/rtopk.h): beside the selections, whose columns are a router's picks.
Argument marshalling only: natively (csrc/rtopk_torch.cpp) in the usual case, through ctypes for the rest.

Logits are [N, E] float32, float16 or bfloat16 tensors on the GPU whose rows are contiguous; work goes to the current stream of their device.  There is
no autograd graph: the forward call returns what the backward call takes."""
from __future__ import annotations

from . import rtopk as _r
from .logits import _given, _gradient, _output, _rows, _type


def rtopk_balance_workspace_bytes(N: int, E: int, dtype, k: int, groups: int = 1) -> int:
    """Device memory that the C entry point can use for such a call; dtype: of the logits, k: picks of a token."""
    return int(_r.load_library().rtopk_balance_workspace_bytes(N, E, _type(dtype), k, groups))


def _picks(cols, N: int, groups: int, device):
    import torch

    if not (isinstance(cols, torch.Tensor) and cols.dim() == 2):
        raise ValueError("cols must be an [N, k] tensor")
    _given(cols, (torch.int32, torch.uint8), (N, cols.shape[1]), device, "cols")
    return cols.data_ptr(), cols.element_size(), cols.shape[1], groups


def rtopk_balance_loss(logits, cols, groups: int = 1, out_loss=None, out_z=None, out_probs=None, out_counts=None, out_rows=None):
    """Balance loss of router logits [N, E] (E up to 1024) and the picked columns [N, k] int32 or uint8, as the selections return them, for each of
    `groups` groups of N / groups consecutive tokens: (loss [groups], z [groups], probs [groups, E], counts [groups, E] int32, rows [groups] int32), the rest
    float32.  loss = E sum_e f_e P_e with the shares f of the picks (counts / their sum) and the mean probabilities P (probs); z: the mean of the squared
    log-sum-exps; rows: tokens that count.  A column outside [0, E) is no pick; a token without any is left out."""
    done = (_r._fast or _r._native()).balance_loss(logits, cols, groups, out_loss, out_z, out_probs, out_counts, out_rows)
    if done is not None:
        return done
    import torch

    x, stream = _rows(logits, "logits")
    N, E, device = x[2], x[3], logits.device
    picks = _picks(cols, N, groups, device)
    if groups < 1:
        _r._check(-2)
    loss = _output(out_loss, torch.float32, (groups,), device, "out_loss")
    z = _output(out_z, torch.float32, (groups,), device, "out_z")
    probs = _output(out_probs, torch.float32, (groups, E), device, "out_probs")
    counts = _output(out_counts, torch.int32, (groups, E), device, "out_counts")
    rows = _output(out_rows, torch.int32, (groups,), device, "out_rows")
    n = rtopk_balance_workspace_bytes(N, E, logits.dtype, cols.shape[1], groups)
    ws = torch.empty((n,), dtype=torch.uint8, device=device) if n > 0 else None
    with torch.cuda.device(device):
        _r._check(_r.load_library().rtopk_balance_loss(*x, *picks, loss.data_ptr(), z.data_ptr(), probs.data_ptr(), counts.data_ptr(), rows.data_ptr(),
                                                       ws.data_ptr() if n > 0 else None, n, stream))
    return loss, z, probs, counts, rows


def rtopk_balance_loss_backward(grad_loss, logits, cols, counts, rows, grad_z=None, grad_vals=None, grad_logits=None):
    """Gradient of rtopk_balance_loss with respect to the logits: [N, E] of their type, from grad_loss [groups] and, if given, grad_z [groups] and the
    gradients of the picked values grad_vals [N, k], all float32.  counts [groups, E] and rows [groups]: what the forward call returned (counts may be sums
    over processes); shares of picks are constants.  grad_logits may be the logits themselves, which are then replaced."""
    done = (_r._fast or _r._native()).balance_loss_backward(grad_loss, logits, cols, counts, rows, grad_z, grad_vals, grad_logits)
    if done is not None:
        return done
    import torch

    x, stream = _rows(logits, "logits")
    N, E, device = x[2], x[3], logits.device
    if not (isinstance(counts, torch.Tensor) and counts.dim() == 2 and counts.shape[0] > 0):
        raise ValueError("counts must be a [groups, E] tensor")
    groups, f32, i32 = counts.shape[0], (torch.float32,), (torch.int32,)
    picks = _picks(cols, N, groups, device)
    _given(counts, i32, (groups, E), device, "counts")
    _given(rows, i32, (groups,), device, "rows")
    _given(grad_loss, f32, (groups,), device, "grad_loss")
    if grad_z is not None:
        _given(grad_z, f32, (groups,), device, "grad_z")
    if grad_vals is not None:
        _given(grad_vals, f32, cols.shape, device, "grad_vals")
    grad = _gradient(grad_logits, logits)
    out, _ = _rows(grad, "grad_logits")
    with torch.cuda.device(device):
        _r._check(_r.load_library().rtopk_balance_loss_backward(
            grad_loss.data_ptr(), grad_z.data_ptr() if grad_z is not None else None, grad_vals.data_ptr() if grad_vals is not None else None, *x, *picks,
            counts.data_ptr(), rows.data_ptr(), out[0], out[4], stream))
    return grad
