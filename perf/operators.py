"""Timed cases of the operators on rows of logits: log probabilities of given tokens with entropy and top alternatives,
distillation from a teacher's top logits, and the gradients of both, through the public Python entry points.

A case is a dict of plain values:
  op        "logprobs" (log probabilities of the given tokens, entropy, log-sum-exp and the `k` top alternatives),
            "logprobs_backward" (gradient of the log probabilities and, with `entropy`, of the entropy),
            "distill" (the loss of each row against the teacher's `k` entries), "distill_backward" (its gradient from the saved
            log-sum-exp), "distill_with_grad" (loss and gradient in one call, the rows' weights known beforehand)
  N, M      rows (positions), columns (vocabulary)
  pad       columns of each stored row beyond M, which belong to no row (the rows' stride is M + pad)
  dtype     "f32", "f16" or "bf16": how the logits are stored, and their gradient
  k         top alternatives (logprobs) or entries of the teacher's list (distill*)
  tokens    given tokens for each row (logprobs*)
  ignored   every so many-th row is one to be left out (token -100, no teacher entry, weight 0); 0: none
  mask      "none", "tail" (the last sixteenth of the columns is -inf: a vocabulary filled up to a round size) or "allowed" (all but
            about one column in 64 are -inf: constrained decoding)
  temperature
  log_probs whether the teacher's entries are log probabilities (distill*), else logits to be normalised over the list
  entropy   whether the entropy has a gradient too (logprobs_backward)

Log probabilities, entropies and losses are 32-bit values, gradients have the logits' type, columns are whole numbers
(equal logits: the lower column first).
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_CELLS = 1 << 30  # of the largest listed case


def _case(op, N, M, dtype, k=0, **more):
    case = dict(op=op, N=N, M=M, dtype=dtype, k=k, pad=0, ignored=0, mask="none", temperature=1.0)
    if op.startswith("logprobs"):
        case["tokens"] = 1
    else:
        case["log_probs"] = False
    if op == "logprobs_backward":
        case["entropy"] = False
    case.update(more)
    return case


def listed():
    return [
        # one token of one sequence, its probability and five alternatives: all latency
        dict(_case("logprobs", 1, 32768, "f32", k=5), name="logprobs_1x32768_f32"),
        # a decoding step of a serving batch, the alternatives that a client may ask for
        dict(_case("logprobs", 64, 131072, "bf16", k=20, temperature=0.7), name="logprobs_64x131072_bf16"),
        # a prompt's positions scored, an odd vocabulary without padding, so that rows start at any element
        dict(_case("logprobs", 8191, 50001, "f16", k=1), name="logprobs_8191x50001_f16"),
        # constrained decoding: few columns are left, some positions are padding
        dict(_case("logprobs", 1000, 32000, "f32", k=8, mask="allowed", ignored=8), name="logprobs_1000x32000_allowed"),
        # a small step of policy training, rewards on log probabilities and on the entropy
        dict(_case("logprobs_backward", 256, 32000, "f32", entropy=True), name="logprobs_bwd_256x32000_f32"),
        # a large one, an eighth of the positions is prompt
        dict(_case("logprobs_backward", 4096, 131072, "bf16", entropy=True, ignored=8), name="logprobs_bwd_4096x131072_bf16"),
        # validation of a student on one short sequence; the vocabulary's rows are padded
        dict(_case("distill", 33, 32003, "f32", k=32, pad=61), name="distill_33x32003_f32"),
        # validation on a batch, the teacher's own log probabilities
        dict(_case("distill", 2048, 131072, "bf16", k=64, log_probs=True), name="distill_2048x131072_bf16"),
        # gradients from outside (the loss goes on into others), softened distributions
        dict(_case("distill_backward", 2048, 65536, "f32", k=100, temperature=2.0), name="distill_bwd_2048x65536_f32"),
        # one short sequence of a training step
        dict(_case("distill_with_grad", 16, 32001, "bf16", k=16), name="distill_step_16x32001_bf16"),
        # a training step at an ordinary vocabulary, in 32 bits
        dict(_case("distill_with_grad", 2048, 50000, "f32", k=100, temperature=2.0), name="distill_step_2048x50000_f32"),
        # a large step at a large vocabulary filled up to a round size
        dict(_case("distill_with_grad", 8192, 131072, "bf16", k=64, mask="tail", ignored=8), name="distill_step_8192x131072_bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the listed ones' ranges: vocabularies of 1000 to 262144 columns, one row to as many as the largest case has cells for."""
    op = rng.choice(("logprobs", "logprobs", "logprobs_backward", "distill", "distill_backward", "distill_with_grad", "distill_with_grad"))
    M = _spread(rng, 1000, 262144)
    shape = rng.randrange(4)  # half of the widths are multiples of 64, a quarter odd
    if shape < 2:
        M = (M + 63) // 64 * 64
    elif shape == 2:
        M |= 1
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    N = _spread(rng, 1, max(1, min(16384, _CELLS * 2 // _BYTES[dtype] // (M + 64))))
    more = dict(pad=rng.choice((0, 0, rng.randrange(1, 64))), ignored=rng.choice((0, 0, 3, 8)), temperature=rng.choice((1.0, 1.0, 0.7, 2.0)))
    if op == "logprobs":
        more.update(k=rng.choice((0, 1, 5, 20, _spread(rng, 1, 128))), tokens=rng.choice((1, 1, 1, 4)), mask=rng.choice(("none", "none", "tail", "allowed")))
    elif op == "logprobs_backward":
        more.update(tokens=rng.choice((1, 1, 4)), entropy=rng.choice((True, False)), mask=rng.choice(("none", "none", "tail")))
    else:
        more.update(k=_spread(rng, 4, 256), log_probs=rng.choice((True, False)), mask=rng.choice(("none", "none", "tail")))
    return _case(op, N, M, dtype, **more)


def _logits(case, gen, scale):
    N, M = case["N"], case["M"]
    x = torch.randn((N, M + case["pad"]), device="cuda", generator=gen, dtype=_DTYPES[case["dtype"]]).mul_(scale).sub_(2)
    if case["mask"] == "tail":
        x[:, M - M // 16:M] = -math.inf
    elif case["mask"] == "allowed":
        x.masked_fill_(torch.rand(x.shape, device="cuda", generator=gen) >= 1 / 64, -math.inf)
        x[:, :M].scatter_(1, torch.randint(0, M, (N, 1), device="cuda", generator=gen), 4.0)  # one column is always left
    return x[:, :M]


def _finite_columns(case):
    return case["M"] - (case["M"] // 16 if case["mask"] == "tail" else 0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    N, k, T = case["N"], case["k"], case["temperature"]
    state = dict(case, logits=_logits(case, gen, 3.0))
    x = state["logits"]
    out = torch.zeros((N, 1), dtype=torch.bool, device="cuda")  # rows to be left out
    if case["ignored"]:
        out[case["ignored"] - 1::case["ignored"]] = True
    if case["op"].startswith("logprobs"):
        G = case["tokens"]
        tokens = torch.randint(0, _finite_columns(case), (N, G), device="cuda", generator=gen)
        if case["mask"] == "allowed":  # the tokens that were drawn are allowed ones
            tokens = torch.topk(x.float(), G, dim=1)[1]
        tokens = tokens.masked_fill(out, -100)
        state["given"] = (tokens[:, 0] if G == 1 else tokens).contiguous()
    else:
        vals, cols = torch.topk(x.float() + torch.randn(x.shape, device="cuda", generator=gen), k, dim=1)
        cols, order = torch.sort(cols, dim=1)
        vals = torch.gather(vals, 1, order)
        if case["log_probs"]:  # nine tenths of the teacher's mass are on the list
            vals = torch.log_softmax(vals / T, 1) + math.log(0.9)
        state["teacher_vals"] = vals.contiguous()
        state["teacher_cols"] = cols.to(torch.int32).masked_fill(out, -1).contiguous()
        if case["op"] == "distill_with_grad":
            state["weights"] = torch.full((N,), 1 / N, device="cuda").masked_fill(out[:, 0], 0.0)
    if case["op"].endswith("_backward"):  # what the forward pass saved, and the gradients that come in
        lse = torch.logsumexp(x.float() / T, 1)
        state["lse"] = lse
        if case["op"] == "logprobs_backward":
            state["grad"] = torch.randn(state["given"].shape, device="cuda", generator=gen)
            if case["entropy"]:
                q = torch.softmax(x.float() / T, 1)
                state["entropy_value"] = lse - (q * (x.float() / T).clamp_(min=-1e30)).sum(1)
                state["grad_entropy"] = torch.randn((N,), device="cuda", generator=gen).mul_(0.1).masked_fill(out[:, 0], 0.0)
        else:
            state["grad"] = torch.randn((N,), device="cuda", generator=gen)
    return state


def _normalised(x, T):
    """x / T less its row's log-sum-exp, and that; a row of nothing but -inf has -inf for both."""
    y = x.float() / T
    top = y.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    lse = torch.log(torch.exp(y - top).sum(1, keepdim=True)) + top
    return torch.where(lse == -math.inf, y, y - lse), lse


def _places(cols, M):
    """Columns as indexes, and which of them count."""
    cols = cols.long()
    valid = (cols >= 0) & (cols < M)
    return torch.where(valid, cols, torch.zeros_like(cols)), valid


def _teacher(state):
    """The teacher's probabilities and their logarithms, zero where an entry does not count."""
    T, vals = state["temperature"], state["teacher_vals"].float()
    cols, valid = _places(state["teacher_cols"], state["M"])
    logp = vals if state["log_probs"] else _normalised(torch.where(valid, vals, torch.full_like(vals, -math.inf)), T)[0]
    valid = valid & (logp > -math.inf)
    return cols, torch.where(valid, torch.exp(logp), torch.zeros_like(logp)), torch.where(valid, logp, torch.zeros_like(logp))


def _distill_loss(state, logq):
    cols, p, logp = _teacher(state)
    return torch.where(p > 0, p * (logp - torch.gather(logq, 1, cols)), torch.zeros_like(p)).sum(1)


def _distill_gradient(state, logq, grad):
    cols, p, _ = _teacher(state)
    g = grad[:, None] / state["temperature"]
    dense = g * p.sum(1, keepdim=True) * torch.exp(logq)
    return dense.scatter_add_(1, cols, -g * p).to(state["logits"].dtype)


def _plain(state):
    op, x, T, M = state["op"], state["logits"], state["temperature"], state["M"]
    if op == "logprobs":
        logq, lse = _normalised(x, T)
        q = torch.exp(logq)
        entropy = -torch.where(q > 0, q * logq, torch.zeros_like(q)).sum(1)
        given = state["given"].view(state["N"], -1)
        cols, valid = _places(given, M)
        logprobs = torch.where(valid, torch.gather(logq, 1, cols), torch.zeros_like(cols, dtype=torch.float32))
        if not state["k"]:
            return logprobs.view(state["given"].shape), entropy, lse[:, 0]
        bits = (x.float() + 0.0).view(torch.int32).long()  # whole numbers in the order of the logits, the lower column first
        bits = torch.where(bits >= 0, bits, -(bits & 0x7fffffff) - 1)
        keys = bits * (1 << 24) + (M - 1 - torch.arange(M, device=x.device))
        top = M - 1 - (torch.topk(keys, state["k"], dim=1)[0] & 0xffffff)
        return logprobs.view(state["given"].shape), entropy, lse[:, 0], torch.gather(logq, 1, top), top.to(torch.int32)
    if op == "logprobs_backward":
        logq = x.float() / T - state["lse"][:, None]
        q = torch.exp(logq)
        given = state["given"].view(state["N"], -1)
        cols, valid = _places(given, M)
        g = torch.where(valid, state["grad"].view(given.shape), torch.zeros_like(cols, dtype=torch.float32))
        dense = -g.sum(1, keepdim=True) * q
        if state["entropy"]:
            dense = dense - state["grad_entropy"][:, None] * torch.where(q > 0, q * (logq + state["entropy_value"][:, None]), torch.zeros_like(q))
        return (dense.scatter_add_(1, cols, g) / T).to(x.dtype)
    if op == "distill":
        logq, lse = _normalised(x, T)
        return _distill_loss(state, logq), lse[:, 0]
    if op == "distill_backward":
        return _distill_gradient(state, x.float() / T - state["lse"][:, None], state["grad"])
    logq, _ = _normalised(x, T)
    return _distill_loss(state, logq), _distill_gradient(state, logq, state["weights"])


def run(state):
    if not own:
        return _plain(state)
    import paper_2409_00822_amd as R

    op, x, T = state["op"], state["logits"], state["temperature"]
    if op == "logprobs":
        return R.rtopk_token_logprobs(x, state["given"], state["k"], T)
    if op == "logprobs_backward":
        if state["entropy"]:
            return R.rtopk_token_logprobs_backward(state["grad"], x, state["given"], state["lse"], T, grad_entropy=state["grad_entropy"],
                                                   entropy=state["entropy_value"])
        return R.rtopk_token_logprobs_backward(state["grad"], x, state["given"], state["lse"], T)
    tv, tc, lp = state["teacher_vals"], state["teacher_cols"], state["log_probs"]
    if op == "distill":
        return R.rtopk_distill(x, tv, tc, T, log_probs=lp)
    if op == "distill_backward":
        return R.rtopk_distill_backward(state["grad"], x, tv, tc, state["lse"], T, log_probs=lp)
    return R.rtopk_distill_with_grad(state["weights"], x, tv, tc, T, log_probs=lp)


def _read_rows(case):
    """Rows that have to be read: a row that is left out has no loss and a gradient of zero whatever its logits are, but an entropy and a
    log-sum-exp."""
    N, every = case["N"], case["ignored"]
    return N - (N // every if every and case["op"] in ("logprobs_backward", "distill_backward", "distill_with_grad") else 0)


def work(case):
    N, M, b, op = case["N"], case["M"], _BYTES[case["dtype"]], case["op"]
    cells = _read_rows(case) * M
    bytes_ = cells * b
    if op == "logprobs":
        return {"bytes": bytes_ + N * (case["tokens"] * (8 + 4) + 8 + 8 * case["k"]), "flops": 6 * cells}
    if op == "logprobs_backward":
        return {"bytes": bytes_ + N * M * b + N * (case["tokens"] * (8 + 4) + 4 + (8 if case["entropy"] else 0)), "flops": (7 if case["entropy"] else 4) * cells}
    bytes_ += N * 8 * case["k"] + 8 * N
    if op == "distill":
        return {"bytes": bytes_, "flops": 4 * cells}
    return {"bytes": bytes_ + N * M * b, "flops": (4 if op == "distill_backward" else 7) * cells}


def _exact_rows(s):
    """The definitions on some rows, in 64 bits, probabilities first."""
    op, T, M = s["op"], s["temperature"], s["M"]
    x = s["logits"].double() / T
    n = x.shape[0]
    row = torch.arange(n, device=x.device)[:, None]
    lse = torch.logsumexp(x, 1)
    if op.startswith("logprobs"):
        given = s["given"].view(n, -1)
        counts = (given >= 0) & (given < M)
        at = given.clamp(0, M - 1)
        q = torch.softmax(x, 1)
        entropy = torch.special.entr(q).sum(1)
        if op == "logprobs":
            logprobs = torch.where(counts, x[row, at] - lse[:, None], 0.0)
            found = [logprobs.view(s["given"].shape), entropy, lse]
            if s["k"]:
                found += [torch.topk(x, s["k"], dim=1)[0] - lse[:, None], None]
            return found
        g = s["grad"].view(n, -1).double() * counts
        mixed = torch.zeros_like(x).index_put_((row.expand_as(at), at), g, accumulate=True) - g.sum(1, keepdim=True) * q
        if s["entropy"]:
            mixed += s["grad_entropy"].double()[:, None] * (torch.special.entr(q) - q * entropy[:, None])
        return [mixed / T]
    cols = s["teacher_cols"].long()
    counts = (cols >= 0) & (cols < M)
    at = cols.clamp(0, M - 1)
    t = s["teacher_vals"].double()
    p = (t.exp() if s["log_probs"] else torch.softmax(t / T, 1)) * counts
    if not s["log_probs"]:
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    loss = (-torch.special.entr(p) - torch.xlogy(p, torch.exp(x[row, at] - lse[:, None]))).sum(1)
    if op == "distill":
        return [loss, lse]
    whole = p.sum(1, keepdim=True) * torch.softmax(x, 1)
    whole.index_put_((row.expand_as(at), at), -p, accumulate=True)
    if op == "distill_backward":
        return [whole * (s["grad"].double()[:, None] / T)]
    return [loss, whole * (s["weights"].double()[:, None] / T)]


def exact(case, seed):
    state = prepare(case, seed)
    step = max(1, (1 << 27) // case["M"])
    per_row = {name for name, v in state.items() if isinstance(v, torch.Tensor)}
    parts = [_exact_rows({name: v[r:r + step] if name in per_row else v for name, v in state.items()}) for r in range(0, case["N"], step)]
    found = [None if p[0] is None else torch.cat(p) for p in zip(*parts)]
    return tuple(found) if len(found) > 1 else found[0]
