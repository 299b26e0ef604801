"""Tokens drawn from rows of logits, and drafted tokens verified against them, with the names of the C ABI (include/rtopk.h).  Argument marshalling
only: natively (csrc/rtopk_torch.cpp) in the usual case, through ctypes for the rest.

Random numbers are inputs, so a call's result is a pure function of its arguments; what decides on a token is computed in 64 bits.  Logits
are float32, float16 or bfloat16 tensors on the GPU whose rows are contiguous; work goes to the current stream of the logits' device."""
from __future__ import annotations

from . import rtopk as _r
from .logits import _given, _output, _rows, _type


def rtopk_verify_workspace_bytes(B: int, G: int, M: int, dtype, draft_logits: bool = False) -> int:
    """Device memory that the C entry points can use for such a call; dtype: of the logits.  G = 0: rtopk_sample_tokens."""
    return int(_r.load_library().rtopk_verify_workspace_bytes(B, G, M, _type(dtype), 1 if draft_logits else 0))


def _random(uniforms, temperature, shape, B: int, device):
    """The C arguments of the random numbers and temperatures."""
    import torch

    per_sequence = isinstance(temperature, torch.Tensor)
    if per_sequence:
        _given(temperature, (torch.float32,), (B,), device, "temperature")
    if uniforms is None and (per_sequence or temperature != 0):
        raise ValueError("random numbers are needed unless the temperature is 0")
    if uniforms is not None:
        _given(uniforms, (torch.float32,), shape, device, "uniforms")
    return (uniforms.data_ptr() if uniforms is not None else None, temperature.data_ptr() if per_sequence else None,
            1.0 if per_sequence else float(temperature))


def _workspace(B: int, G: int, M: int, dtype, draft_logits: bool, device):
    import torch

    n = rtopk_verify_workspace_bytes(B, G, M, dtype, draft_logits)
    if n == 0:
        return None, 0, None
    w = torch.empty((n,), dtype=torch.uint8, device=device)
    return w.data_ptr(), n, w


def _tokens_out(t, dtypes, shape, device):
    import torch

    if t is None:
        return torch.empty(tuple(shape), dtype=dtypes[0], device=device)
    return _given(t, dtypes, shape, device, "out_tokens")


def _sequences(x, name: str):
    """B, positions, M and the strides of [B, positions, M] logits."""
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 3):
        raise ValueError(f"{name} must be a 3-D tensor on the GPU")
    B, P, M = x.shape
    seq, pos = x.stride(0) if B > 1 else M, x.stride(1) if P > 1 else M
    if (x.stride(2) != 1 and M > 1) or seq < M or pos < M:
        raise ValueError(f"the rows of {name} must be contiguous and must not overlap")
    return B, P, M, seq, pos


def rtopk_sample_tokens(logits, uniforms, temperature=1.0, out_tokens=None):
    """A token of each row of logits [N, M], drawn from softmax(logits / temperature) by uniforms [N] float32 in [0, 1): the lowest column that the
    cumulated probability passes the number at.  temperature: a number, or [N] float32, one for each row; 0: the largest logit, the lowest column of equal
    ones (uniforms may be None where it is the number 0).  Returns [N] int64 (or out_tokens' int32); -1 for a row with nothing but -inf, a NaN or +inf."""
    done = (_r._fast or _r._native()).sample_tokens(logits, uniforms, temperature, out_tokens)
    if done is not None:
        return done
    import torch

    rows, stream = _rows(logits, "logits")
    N, M, device = rows[2], rows[3], logits.device
    random = _random(uniforms, temperature, (N,), N, device)
    out = _tokens_out(out_tokens, (torch.int64, torch.int32), (N,), device)
    ws, ws_bytes, _keep = _workspace(N, 0, M, logits.dtype, False, device)
    with torch.cuda.device(device):
        _r._check(_r.load_library().rtopk_sample_tokens(*rows, *random, out.data_ptr(), out.element_size(), ws, ws_bytes, stream))
    return out


def rtopk_verify_drafts(target_logits, drafts, uniforms, draft_logits=None, temperature=1.0, out_tokens=None, out_accepted=None):
    """Accepts drafted tokens [B, G] (int32 or int64, G up to 128; the first one outside [0, M) ends a sequence's drafts) against target_logits
    [B, G + 1, M] by uniforms [B, G + 1] float32 in [0, 1), and draws one more token: (tokens [B, G + 1] of the drafts' type, the accepted drafts, the drawn
    token, -1 behind it; accepted [B] int32).  A draft is accepted if u q < p, with q from draft_logits [B, G, M] (None: q = 1, a draft that was looked
    up); the first rejected one is replaced by a draw by u_G from max(p - q, 0), and behind accepted ones the draw is from the next row.
    temperature: a number, or [B] float32, of target and draft alike; 0: the largest logits.  Strides between sequences and positions are free."""
    done = (_r._fast or _r._native()).verify_drafts(target_logits, drafts, uniforms, draft_logits, temperature, out_tokens, out_accepted)
    if done is not None:
        return done
    import torch

    B, P, M, seq, pos = _sequences(target_logits, "target_logits")
    device, dtype = target_logits.device, _type(target_logits.dtype)
    G = P - 1
    if G < 0:
        raise ValueError("target_logits must have a row more than there are drafts")
    _given(drafts, (torch.int32, torch.int64), (B, G), device, "drafts")
    random = _random(uniforms, temperature, (B, G + 1), B, device)
    draft = (None, 0, 0)
    if draft_logits is not None:
        b, g, m, draft_seq, draft_pos = _sequences(draft_logits, "draft_logits")
        if (b, g, m) != (B, G, M) or draft_logits.dtype != target_logits.dtype or draft_logits.device != device:
            raise ValueError("draft_logits must be [B, G, M] of the target's type and device")
        draft = (draft_logits.data_ptr() if draft_logits.numel() else None, draft_seq, draft_pos)
    out = _tokens_out(out_tokens, (drafts.dtype,), (B, G + 1), device)
    accepted = _output(out_accepted, torch.int32, (B,), device, "out_accepted")
    ws, ws_bytes, _keep = _workspace(B, G, M, target_logits.dtype, draft[0] is not None, device)
    with torch.cuda.device(device):
        _r._check(_r.load_library().rtopk_verify_drafts(
            target_logits.data_ptr(), draft[0], dtype, B, G, M, seq, pos, draft[1], draft[2], drafts.data_ptr(), drafts.element_size(), *random,
            out.data_ptr(), accepted.data_ptr(), ws, ws_bytes, torch.cuda.current_stream(device).cuda_stream))
    return out, accepted
