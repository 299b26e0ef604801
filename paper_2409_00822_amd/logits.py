"""Operators on rows of logits, with the names of the C ABI (include/rtopk.h): log probabilities of given tokens with entropy and top
alternatives, distillation from a teacher's top logits, and the gradients of both.  Argument marshalling only: natively
(csrc/rtopk_torch.cpp) in the usual case, through ctypes for the rest.

Logits are [N, M] float32, float16 or bfloat16 tensors on the GPU whose rows are contiguous (a slice of a padded vocabulary is fine); results
and sums are float32, gradients have the logits' type.  There is no autograd graph: the forward calls return what the backward calls take.
Columns, losses and gradients are in the order of the arguments; work goes to the current stream of the logits' device."""
from __future__ import annotations

from . import rtopk as _r


def rtopk_logits_workspace_bytes(N: int, M: int, dtype, k: int = 0) -> int:
    """Device memory that the C entry points can use for such a call; dtype: of the logits, k: alternatives."""
    return int(_r.load_library().rtopk_logits_workspace_bytes(N, M, _type(dtype), k))


def _type(dtype) -> int:
    import torch

    found = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}.get(dtype)
    if found is None:
        raise ValueError(f"logits and teacher values are float32, float16 or bfloat16, not {dtype}")
    return found


def _rows(x, name: str):
    """The C arguments of rows of logits, and their stream."""
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 2):
        raise ValueError(f"{name} must be a 2-D tensor on the GPU")
    dtype = _type(x.dtype)
    N, M = x.shape
    stride = x.stride(0) if N > 1 else M
    if (x.stride(1) != 1 and M > 1) or stride < M:
        raise ValueError(f"the rows of {name} must be contiguous and must not overlap")
    return (x.data_ptr(), dtype, N, M, stride), torch.cuda.current_stream(x.device).cuda_stream


def _given(t, dtypes, shape, device, name: str):
    """Checks an input and returns it."""
    import torch

    if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype in dtypes and tuple(t.shape) == tuple(shape) and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {list(shape)} tensor of {' or '.join(str(d) for d in dtypes)} on the logits' device")
    return t


def _output(t, dtype, shape, device, name: str):
    """The caller's output, checked, or a new one."""
    import torch

    if t is None:
        return torch.empty(tuple(shape), dtype=dtype, device=device)
    return _given(t, (dtype,), shape, device, name)


def _gradient(t, x):
    """The caller's rows for the gradient, checked, or new ones."""
    import torch

    if t is None:
        return torch.empty(tuple(x.shape), dtype=x.dtype, device=x.device)
    if not (isinstance(t, torch.Tensor) and t.device == x.device and t.dtype == x.dtype and t.shape == x.shape):
        raise ValueError("grad_logits must have the logits' shape, type and device")
    return t


def _workspace(N: int, M: int, dtype, k: int, device):
    import torch

    n = rtopk_logits_workspace_bytes(N, M, dtype, k) if 0 <= k <= 128 else 0
    if n == 0:
        return None, 0, None
    w = torch.empty((n,), dtype=torch.uint8, device=device)
    return w.data_ptr(), n, w


def _tokens(tokens, N: int, device):
    import torch

    if not (isinstance(tokens, torch.Tensor) and tokens.dim() in (1, 2)):
        raise ValueError("tokens must be an [N] or [N, G] tensor")
    shape = (N,) if tokens.dim() == 1 else (N, tokens.shape[1])
    _given(tokens, (torch.int32, torch.int64), shape, device, "tokens")
    return tokens.data_ptr(), tokens.element_size(), 1 if tokens.dim() == 1 else tokens.shape[1]


def _teacher(vals, cols, log_probs, N: int, device):
    import torch

    if not (isinstance(vals, torch.Tensor) and vals.dim() == 2):
        raise ValueError("teacher_vals must be an [N, k] tensor")
    dtype = _type(vals.dtype)
    _given(vals, (vals.dtype,), (N, vals.shape[1]), device, "teacher_vals")
    _given(cols, (torch.int32,), (N, vals.shape[1]), device, "teacher_cols")
    return vals.data_ptr(), dtype, cols.data_ptr(), vals.shape[1], 1 if log_probs else 0


def rtopk_token_logprobs(logits, tokens, k: int = 0, temperature: float = 1.0, out_logprobs=None, out_entropy=None, out_lse=None,
                         out_top_logprobs=None, out_top_cols=None):
    """Log probabilities of `tokens` ([N] or [N, G], int32 or int64; outside [0, M): left out, 0) under softmax(logits / temperature), and
    each row's entropy and log-sum-exp: (logprobs of tokens' shape, entropy [N], lse [N]).  With k > 0 (up to 128) also
    the k largest logits' log probabilities [N, k], largest first, equal ones by column, and their columns [N, k] int32."""
    done = (_r._fast or _r._native()).token_logprobs(logits, tokens, k, temperature, out_logprobs, out_entropy, out_lse, out_top_logprobs,
                                                     out_top_cols)
    if done is not None:
        return done
    import torch

    rows, stream = _rows(logits, "logits")
    N, M, device = rows[2], rows[3], logits.device
    given = _tokens(tokens, N, device)
    if k < 0:
        _r._check(-2)
    if k == 0 and (out_top_logprobs is not None or out_top_cols is not None):
        raise ValueError("outputs for alternatives need k > 0")
    logprobs = _output(out_logprobs, torch.float32, tokens.shape, device, "out_logprobs")
    entropy = _output(out_entropy, torch.float32, (N,), device, "out_entropy")
    lse = _output(out_lse, torch.float32, (N,), device, "out_lse")
    top = []
    if k > 0:
        top = [_output(out_top_logprobs, torch.float32, (N, k), device, "out_top_logprobs"),
               _output(out_top_cols, torch.int32, (N, k), device, "out_top_cols")]
    ws, ws_bytes, _keep = _workspace(N, M, logits.dtype, k, device)
    _r._check(_r.load_library().rtopk_token_logprobs(
        *rows, *given, k, float(temperature), logprobs.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
        top[0].data_ptr() if top else None, top[1].data_ptr() if top else None, ws, ws_bytes, stream))
    return (logprobs, entropy, lse, *top)


def rtopk_token_logprobs_backward(grad_logprobs, logits, tokens, lse, temperature: float = 1.0, grad_entropy=None, entropy=None,
                                  grad_logits=None):
    """Gradient of rtopk_token_logprobs with respect to the logits, from the gradient of its log probabilities (tokens' shape) and, if given, of
    its entropy ([N], with the entropy itself).  `lse`: what the forward call returned at the same temperature.  Returns [N, M] of
    the logits' type; grad_logits may be the logits themselves, which are then replaced."""
    done = (_r._fast or _r._native()).token_logprobs_backward(grad_logprobs, logits, tokens, lse, temperature, grad_entropy, entropy, grad_logits)
    if done is not None:
        return done
    import torch

    rows, stream = _rows(logits, "logits")
    N, device = rows[2], logits.device
    given = _tokens(tokens, N, device)
    f32 = (torch.float32,)
    _given(grad_logprobs, f32, tokens.shape, device, "grad_logprobs")
    _given(lse, f32, (N,), device, "lse")
    if grad_entropy is not None:
        _given(grad_entropy, f32, (N,), device, "grad_entropy")
        _given(entropy, f32, (N,), device, "entropy")
    grad = _gradient(grad_logits, logits)
    out, _ = _rows(grad, "grad_logits")
    _r._check(_r.load_library().rtopk_token_logprobs_backward(
        grad_logprobs.data_ptr(), grad_entropy.data_ptr() if grad_entropy is not None else None, *rows, *given, lse.data_ptr(),
        entropy.data_ptr() if grad_entropy is not None else None, float(temperature), out[0], out[4], stream))
    return grad


def rtopk_distill(logits, teacher_vals, teacher_cols, temperature: float = 1.0, log_probs: bool = False, out_loss=None, out_lse=None):
    """Each row's distillation loss sum_j p_j (ln p_j - ln q_(c_j)) against the teacher's k entries (teacher_vals [N, k] of any of the three
    types, teacher_cols [N, k] int32, up to 1024; a column outside [0, M) or a value of -inf: no entry), and its log-sum-exp: (loss [N], lse [N]).
    q = softmax(logits / temperature); p = softmax(teacher_vals / temperature) over the entries or, with log_probs,
    exp(teacher_vals).  A row without entries has loss 0.  The gradient is with respect to the logits: factors like
    temperature ** 2 are the caller's."""
    done = (_r._fast or _r._native()).distill(logits, teacher_vals, teacher_cols, temperature, log_probs, out_loss, out_lse)
    if done is not None:
        return done
    import torch

    rows, stream = _rows(logits, "logits")
    N, M, device = rows[2], rows[3], logits.device
    teacher = _teacher(teacher_vals, teacher_cols, log_probs, N, device)
    loss = _output(out_loss, torch.float32, (N,), device, "out_loss")
    lse = _output(out_lse, torch.float32, (N,), device, "out_lse")
    ws, ws_bytes, _keep = _workspace(N, M, logits.dtype, 0, device)
    _r._check(_r.load_library().rtopk_distill(*rows, *teacher, float(temperature), loss.data_ptr(), lse.data_ptr(), ws, ws_bytes, stream))
    return loss, lse


def rtopk_distill_backward(grad_loss, logits, teacher_vals, teacher_cols, lse, temperature: float = 1.0, log_probs: bool = False,
                           grad_logits=None):
    """Gradient of rtopk_distill's loss with respect to the logits, from grad_loss [N] and the `lse` it returned: [N, M] of the logits' type.
    grad_logits may be the logits themselves, which are then replaced."""
    done = (_r._fast or _r._native()).distill_backward(grad_loss, logits, teacher_vals, teacher_cols, lse, temperature, log_probs, grad_logits)
    if done is not None:
        return done
    import torch

    rows, stream = _rows(logits, "logits")
    N, device = rows[2], logits.device
    teacher = _teacher(teacher_vals, teacher_cols, log_probs, N, device)
    _given(grad_loss, (torch.float32,), (N,), device, "grad_loss")
    _given(lse, (torch.float32,), (N,), device, "lse")
    grad = _gradient(grad_logits, logits)
    out, _ = _rows(grad, "grad_logits")
    _r._check(_r.load_library().rtopk_distill_backward(grad_loss.data_ptr(), *rows, *teacher, lse.data_ptr(), float(temperature), out[0], out[4],
                                                       stream))
    return grad


def rtopk_distill_with_grad(weights, logits, teacher_vals, teacher_cols, temperature: float = 1.0, log_probs: bool = False, out_loss=None,
                            grad_logits=None):
    """rtopk_distill's loss and, for weights [N] known beforehand (1 / N for a mean), the gradient of sum_n weights_n loss_n in one call:
    (loss [N], gradient [N, M] of the logits' type).  The loss is not weighted.  grad_logits may be the logits themselves."""
    done = (_r._fast or _r._native()).distill_with_grad(weights, logits, teacher_vals, teacher_cols, temperature, log_probs, out_loss, grad_logits)
    if done is not None:
        return done
    import torch

    rows, stream = _rows(logits, "logits")
    N, M, device = rows[2], rows[3], logits.device
    teacher = _teacher(teacher_vals, teacher_cols, log_probs, N, device)
    _given(weights, (torch.float32,), (N,), device, "weights")
    loss = _output(out_loss, torch.float32, (N,), device, "out_loss")
    grad = _gradient(grad_logits, logits)
    out, _ = _rows(grad, "grad_logits")
    ws, ws_bytes, _keep = _workspace(N, M, logits.dtype, 0, device)
    _r._check(_r.load_library().rtopk_distill_with_grad(weights.data_ptr(), *rows, *teacher, float(temperature), loss.data_ptr(), out[0], out[4], ws,
                                                        ws_bytes, stream))
    return loss, grad
