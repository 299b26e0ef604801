"""Timed cases of tokens drawn from rows of logits, drafted tokens verified against them, and of a router's balance loss with its gradient,
through the public Python entry points.

A case is a dict of plain values:
  op        "sample" (one token of each row, drawn by a given random number), "verify" (drafted tokens of each sequence accepted or rejected
            by given random numbers, and one more token drawn), "balance" (balance loss, router z loss, mean probabilities and picks of each
            expert), "balance_backward" (the gradient of both losses, and of the picked values, with respect to the router's logits)
  dtype     "f32", "f16" or "bf16": how the logits are stored, and their gradient
sample:
  N, M, pad    rows, columns (vocabulary), columns of each stored row beyond M that belong to no row
  temperature  a number (0: the largest logit), or "mixed": each sequence has its own, some of them 0
verify:
  B, G, M, pad   sequences, drafted tokens of each, columns
  temperature    as above
  draft          "logits": the draft model's logits are given, at `noise` standard deviations from the target's; "none": the drafts were
                 looked up, and stand for themselves
  noise          (of drafted logits)
  ragged         whether sequences have fewer drafts than G, at random from none to all
balance, balance_backward:
  N, E, k, groups   tokens, experts, picks of each token, groups of tokens (sequences) that are balanced each by itself
  ignored           every so many-th token is padding (its picks are -1); 0: none
  bytes             of a picked column: 4 (int32) or 1 (uint8)
  picked            whether the picked values have a gradient, too (balance_backward)

Random numbers are inputs.  Tokens and picks are whole numbers; what a token depends on is computed in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_TEMPERATURES = (0.0, 0.7, 1.0, 1.0, 1.3)  # of "mixed"
_LEAST_MASS = 2.0**-40  # of a residual distribution: below it target and draft are the same
_VERIFY_CELLS = 256 * 15 * 131072  # of the largest listed case, 16-bit logits


def _sample(N, M, dtype, temperature=1.0, pad=0):
    return dict(op="sample", N=N, M=M, dtype=dtype, temperature=temperature, pad=pad)


def _verify(B, G, M, dtype, draft="logits", temperature=1.0, noise=0.6, ragged=False, pad=0):
    return dict(op="verify", B=B, G=G, M=M, dtype=dtype, draft=draft, temperature=temperature, noise=noise, ragged=ragged, pad=pad)


def _balance(op, N, E, k, dtype, groups=1, ignored=0, bytes=4, picked=False):
    return dict(op=op, N=N, E=E, k=k, dtype=dtype, groups=groups, ignored=ignored, bytes=bytes, picked=picked)


def listed():
    return [
        # the next token of one sequence: all latency
        dict(_sample(1, 32768, "f32", temperature=0.7), name="sample_1x32768_f32"),
        # a decoding step of a serving batch, each sequence with its own temperature
        dict(_sample(64, 131072, "bf16", temperature="mixed"), name="sample_64x131072_bf16"),
        # many continuations of one prompt, an odd vocabulary
        dict(_sample(2047, 50001, "f16"), name="sample_2047x50001_f16"),
        # one sequence with four drafts: all latency
        dict(_verify(1, 4, 32000, "f32", temperature=0.7), name="verify_1x4x32000_f32"),
        # a serving batch, each sequence with its own temperature and number of drafts
        dict(_verify(32, 5, 131072, "bf16", temperature="mixed", ragged=True), name="verify_32x5x131072_bf16"),
        # the same with drafts looked up in the prompt, an odd vocabulary in padded rows
        dict(_verify(64, 3, 50001, "f16", draft="none", pad=15), name="verify_64x3x50001_lookup"),
        # a large batch with long drafts
        dict(_verify(256, 7, 131072, "bf16"), name="verify_256x7x131072_bf16"),
        # the router of one decoding step of a small model
        dict(_balance("balance", 33, 8, 2, "f32"), name="balance_33x8_f32"),
        # a training step's tokens over many experts, each sequence balanced by itself, an eighth is padding
        dict(_balance("balance", 262144, 256, 8, "bf16", groups=64, ignored=8), name="balance_262144x256_bf16"),
        # an ordinary step, byte columns, gradients of the picked values too
        dict(_balance("balance_backward", 16384, 64, 6, "f32", bytes=1, picked=True), name="balance_bwd_16384x64_f32"),
        # a number of experts that fills no lanes, odd numbers of tokens
        dict(_balance("balance_backward", 100002, 60, 4, "f16", groups=6), name="balance_bwd_100002x60_f16"),
        # a large step
        dict(_balance("balance_backward", 1 << 20, 128, 8, "bf16", ignored=8, picked=True), name="balance_bwd_1048576x128_bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def _vocabulary(rng):
    M = _spread(rng, 1000, 262144)
    shape = rng.randrange(4)  # half of the widths are multiples of 64, a quarter odd
    return (M + 63) // 64 * 64 if shape < 2 else (M | 1 if shape == 2 else M)


def draw(rng):
    """Another case of the listed ones' ranges: vocabularies of 1000 to 262144 columns, 4 to 512 experts, one row to as many as the largest cases have."""
    op = rng.choice(("sample", "verify", "verify", "verify", "balance", "balance_backward", "balance_backward"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    temperature = rng.choice((1.0, 0.7, 1.5, "mixed", "mixed", 0.0))
    pad = rng.choice((0, 0, rng.randrange(1, 64)))
    if op == "sample":
        M = _vocabulary(rng)
        return _sample(_spread(rng, 1, min(4096, _VERIFY_CELLS * 2 // _BYTES[dtype] // (M + 64))), M, dtype, temperature, pad)
    if op == "verify":
        M, G = _vocabulary(rng), rng.randrange(1, 9)
        B = _spread(rng, 1, min(512, _VERIFY_CELLS * 2 // _BYTES[dtype] // ((2 * G + 1) * (M + 64))))
        return _verify(B, G, M, dtype, rng.choice(("logits", "logits", "none")), temperature, rng.choice((0.3, 0.6, 1.0)), rng.choice((True, False)), pad)
    E = rng.choice((8, 16, 32, 64, 128, 256, _spread(rng, 4, 512)))
    k = rng.randrange(1, min(E, 12) + 1)
    groups = rng.choice((1, 1, _spread(rng, 2, 128)))
    most = (1 << 27) * 2 // _BYTES[dtype] // (E + 4 * k)
    L = _spread(rng, 1, max(1, most // groups))
    ignored = rng.choice((0, 0, 3, 8))
    return _balance(op, groups * L, E, k, dtype, groups, ignored, 1 if E <= 255 and rng.random() < 0.3 else 4, op == "balance_backward" and rng.random() < 0.6)


def _padded(shape, pad, dtype, gen, scale, shift):
    x = torch.randn((*shape[:-1], shape[-1] + pad), device="cuda", generator=gen, dtype=dtype)
    return x.mul_(scale).add_(shift)[..., :shape[-1]]


def _temperatures(case, rows, gen):
    """What a call takes: a number, or one for each sequence."""
    if case["temperature"] != "mixed":
        return case["temperature"]
    some = torch.tensor(_TEMPERATURES, device="cuda")
    return some[torch.randint(0, len(_TEMPERATURES), (rows,), device="cuda", generator=gen)].contiguous()


def _drawn(x, T, gen):
    """A token of each row [..., M], by one random number for each column; T broadcasts."""
    noise = torch.rand(x.shape, device="cuda", generator=gen).clamp_(min=1e-30).log_().neg_().clamp_(min=1e-30).log_().neg_()
    return (x.float() + noise * T).argmax(-1)


def _prepare_verify(case, gen):
    B, G, M, dtype = case["B"], case["G"], case["M"], _DTYPES[case["dtype"]]
    T = _temperatures(case, B, gen)
    T_rows = T[:, None, None] if isinstance(T, torch.Tensor) else T
    target = _padded((B, G + 1, M), case["pad"], dtype, gen, 3.0, -2.0)
    state = dict(case, target=target, temperature=T, draft_logits=None)
    if case["draft"] == "logits":
        draft = torch.empty((B, G, M + case["pad"]), device="cuda", dtype=dtype)[..., :M]
        draft.copy_(target[:, :G] + case["noise"] * torch.randn((B, G, M), device="cuda", generator=gen, dtype=dtype))
        state["draft_logits"] = draft
        drafts = _drawn(draft, T_rows, gen)
    else:  # two thirds of what was looked up are likely tokens
        drafts = torch.randint(0, M, (B, G), device="cuda", generator=gen)
        hit = torch.rand((B, G), device="cuda", generator=gen) < 0.67
        lse = torch.logsumexp(target[:, :G].float(), -1)
        lifted = lse + 4 * torch.rand((B, G), device="cuda", generator=gen)
        at = drafts[..., None]
        target[:, :G].scatter_(2, at, torch.where(hit[..., None], lifted[..., None].to(dtype), target[:, :G].gather(2, at)))
    if case["ragged"]:
        count = torch.randint(0, G + 1, (B, 1), device="cuda", generator=gen)
        drafts = drafts.masked_fill(torch.arange(G, device="cuda") >= count, -1)
    state["drafts"] = drafts.contiguous()
    state["uniforms"] = torch.rand((B, G + 1), device="cuda", generator=gen)
    return state


def _prepare_balance(case, gen):
    N, E, k = case["N"], case["E"], case["k"]
    x = torch.randn((N, E), device="cuda", generator=gen)
    x += 0.7 * torch.randn((E,), device="cuda", generator=gen)  # some experts are liked better
    state = dict(case, logits=x.to(_DTYPES[case["dtype"]]))
    cols = torch.topk(state["logits"].float(), k, dim=1)[1].sort(dim=1)[0]
    if case["ignored"]:
        cols[case["ignored"] - 1::case["ignored"]] = -1
    state["cols"] = (cols.to(torch.uint8) if case["bytes"] == 1 else cols.to(torch.int32)).contiguous()
    if case["op"] == "balance_backward":  # what the forward pass gave, and the gradients that come in
        state["counts"], state["rows"] = _picks(state)
        scale = 16.0 * N / case["groups"] if case["dtype"] == "f16" else 1.0  # of the loss, as training in half precision has it
        state["grad_loss"] = torch.rand((case["groups"],), device="cuda", generator=gen).add_(0.5).mul_(0.01 * scale)
        state["grad_z"] = torch.full((case["groups"],), 0.001 * scale, device="cuda")
        state["grad_picked"] = torch.randn((N, k), device="cuda", generator=gen).mul_(scale / N) if case["picked"] else None
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "verify":
        return _prepare_verify(case, gen)
    if case["op"] != "sample":
        return _prepare_balance(case, gen)
    x = _padded((case["N"], case["M"]), case["pad"], _DTYPES[case["dtype"]], gen, 3.0, -2.0)
    return dict(case, logits=x, temperature=_temperatures(case, case["N"], gen), uniforms=torch.rand((case["N"],), device="cuda", generator=gen))


def _distribution(x, T):
    """softmax(x / T) of rows [n, ..., M] in 64 bits; T [n] 64-bit, 0: all on the largest logit, the lowest of equal ones."""
    x = x.double()
    T = T.view(-1, *([1] * (x.dim() - 1)))
    top = x.amax(-1, keepdim=True)
    e = torch.exp((x - top) / torch.where(T > 0, T, torch.ones_like(T)))
    p = e / e.sum(-1, keepdim=True)
    if bool((T == 0).any()):
        at = torch.arange(x.shape[-1], device=x.device)
        first = torch.where(x == top, at, torch.full_like(at, x.shape[-1])).amin(-1, keepdim=True)
        p = torch.where(T > 0, p, (at == first).double())
    return p


def _temperature_rows(T, n):
    return T.double() if isinstance(T, torch.Tensor) else torch.full((n,), T, dtype=torch.float64, device="cuda")


def _pick(w, u):
    """The first column of each row [n, M] whose cumulated weight is beyond u of all."""
    total = w.cumsum(1)
    token = (total <= u.double()[:, None] * total[:, -1:]).sum(1)
    at = torch.arange(w.shape[1], device=w.device)
    last = torch.where(w > 0, at, torch.full_like(at, -1)).amax(1)
    return torch.minimum(token, last)


def _plain_verify(s):
    B, G, M, u = s["B"], s["G"], s["M"], s["uniforms"].double()
    T = _temperature_rows(s["temperature"], B)
    at = torch.arange(M, device="cuda")
    drafts = s["drafts"]
    counts = ((drafts >= 0) & (drafts < M)).long().cumprod(1)
    d = torch.where(counts > 0, drafts, torch.zeros_like(drafts))
    p = _distribution(s["target"], T)
    certain = T[:, None, None] == 0  # of the draft: it stands for itself
    if s["draft_logits"] is None:
        q = (at == d[..., None]).double()
    else:
        q = _distribution(s["draft_logits"], T)
        if bool(certain.any()):
            q = torch.where(certain, (at == d[..., None]).double(), q)
    p_d = p[:, :G].gather(2, d[..., None])[..., 0]
    q_d = q.gather(2, d[..., None])[..., 0]
    accepted = ((u[:, :G] * q_d < p_d).long() * counts).cumprod(1).sum(1)
    rejects = accepted < counts.sum(1)
    row = torch.arange(B, device="cuda")
    p_n = p[row, accepted]
    w = (p_n - q[row, torch.clamp(accepted, max=G - 1)]).clamp(min=0)
    w = torch.where((rejects & (w.sum(1) > _LEAST_MASS))[:, None], w, p_n)
    token = _pick(w, u[:, G])
    place = torch.arange(G + 1, device="cuda")
    tokens = torch.cat([d, torch.zeros_like(d[:, :1])], 1)
    tokens = torch.where(place < accepted[:, None], tokens, torch.where(place == accepted[:, None], token[:, None], torch.full_like(tokens, -1)))
    return tokens, accepted.to(torch.int32)


def _picks(s):
    """How often each expert of each group was picked, and the group's tokens that are none of padding."""
    N, E, groups = s["N"], s["E"], s["groups"]
    cols = s["cols"].long().view(groups, -1)
    valid = (cols >= 0) & (cols < E)
    counts = torch.zeros((groups, E + 1), dtype=torch.int64, device="cuda")
    counts.scatter_add_(1, torch.where(valid, cols, torch.full_like(cols, E)), torch.ones_like(cols))
    rows = valid.view(groups, N // groups, -1).any(2).sum(1)
    return counts[:, :E].to(torch.int32).contiguous(), rows.to(torch.int32)


def _router(s):
    """Probabilities and log-sum-exp of each token by groups, 0 for padding, and which tokens count."""
    x = s["logits"].float().view(s["groups"], -1, s["E"])
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    cols = s["cols"].long().view(*x.shape[:2], -1)
    valid = ((cols >= 0) & (cols < s["E"])).any(-1, keepdim=True)
    zero = torch.zeros((), device=x.device)
    return torch.where(valid, e / total, zero), torch.where(valid, torch.log(total) + top, zero), valid


def _plain_balance(s):
    E = s["E"]
    counts, rows = _picks(s)
    p, lse, _ = _router(s)
    n = rows.double().clamp(min=1)[:, None]
    mean = p.sum(1, dtype=torch.float64) / n
    share = counts.double() / counts.sum(1, keepdim=True).clamp(min=1)
    z = (lse * lse).sum(1, dtype=torch.float64) / n
    return (E * (share * mean).sum(1)).float(), z[:, 0].float(), mean.float(), counts, rows


def _plain_balance_backward(s):
    E = s["E"]
    p, lse, _ = _router(s)
    n = s["rows"].float().clamp(min=1)[:, None]
    share = s["counts"].float() / s["counts"].sum(1, keepdim=True).clamp(min=1)
    w = (E * s["grad_loss"][:, None] * share / n)[:, None]
    grad = p * (w - (p * w).sum(-1, keepdim=True) + 2 * (s["grad_z"][:, None, None] / n[..., None]) * lse)
    grad = grad.view(s["N"], E)
    if s["grad_picked"] is not None:
        cols = s["cols"].long()
        valid = (cols >= 0) & (cols < E)
        grad.scatter_add_(1, torch.where(valid, cols, torch.zeros_like(cols)), torch.where(valid, s["grad_picked"], torch.zeros_like(s["grad_picked"])))
    return grad.to(s["logits"].dtype)


def _plain(s):
    if s["op"] == "sample":
        return _pick(_distribution(s["logits"], _temperature_rows(s["temperature"], s["N"])), s["uniforms"])
    if s["op"] == "verify":
        return _plain_verify(s)
    return _plain_balance(s) if s["op"] == "balance" else _plain_balance_backward(s)


def run(state):
    if not own:
        return _plain(state)
    import paper_2409_00822_amd as R

    if state["op"] == "sample":
        return R.rtopk_sample_tokens(state["logits"], state["uniforms"], state["temperature"])
    if state["op"] == "verify":
        return R.rtopk_verify_drafts(state["target"], state["drafts"], state["uniforms"], state["draft_logits"], state["temperature"])
    if state["op"] == "balance":
        return R.rtopk_balance_loss(state["logits"], state["cols"], state["groups"])
    return R.rtopk_balance_loss_backward(state["grad_loss"], state["logits"], state["cols"], state["counts"], state["rows"], grad_z=state["grad_z"],
                                         grad_vals=state["grad_picked"])


def _expected_positions(case):
    """How many of a sequence's positions are looked at on average until one is rejected: rows of the target, rows of the draft.

    Where draft logits are the target's with Gaussian noise of s (in units of the temperature), a draft is accepted with probability
    sum min(p, q) = erfc(s / sqrt 8); of the looked up ones with about 0.6.  Of sequences at temperature 0 about half are taken."""
    T = 1.0 if case["temperature"] == "mixed" else case["temperature"]
    if case["draft"] == "none":
        a = 0.6
    else:
        a = math.erfc(case["noise"] / T / math.sqrt(8)) if T > 0 else 0.5
    lengths = range(case["G"] + 1) if case["ragged"] else [case["G"]]
    target = sum(sum(a**i for i in range(g + 1)) for g in lengths) / len(lengths)
    draft = sum(sum(a**i for i in range(g)) for g in lengths) / len(lengths)
    if case["temperature"] == "mixed":
        draft *= 1 - _TEMPERATURES.count(0.0) / len(_TEMPERATURES)
    return target, draft if case["draft"] == "logits" and case["temperature"] != 0 else 0.0


def work(case):
    b = _BYTES[case["dtype"]]
    if case["op"] == "sample":
        cells = case["N"] * case["M"]
        return {"bytes": cells * b + case["N"] * 12, "flops": 3 * cells}
    if case["op"] == "verify":
        cells = sum(_expected_positions(case)) * case["B"] * case["M"]
        return {"bytes": int(cells * b + case["B"] * ((case["G"] + 1) * 12 + case["G"] * 8 + 4)), "flops": int(3 * cells)}
    N, E, k = case["N"], case["E"], case["k"]
    left_out = N // case["ignored"] if case["ignored"] else 0
    cells, picks = (N - left_out) * E, N * k * case["bytes"]
    if case["op"] == "balance":
        return {"bytes": cells * b + picks + case["groups"] * (8 * E + 12), "flops": 6 * cells}
    return {"bytes": cells * b + N * E * b + picks + (4 * N * k if case["picked"] else 0) + case["groups"] * (4 * E + 12), "flops": 9 * cells}


def _exact_weights(x, T):
    """Relative probabilities of one row of 64-bit logits, largest 1."""
    if T == 0:
        w = torch.zeros_like(x)
        w[torch.nonzero(x == x.max())[0, 0]] = 1
        return w
    return torch.exp2((x - x.max()) * (math.log2(math.e) / T))


def _exact_pick(w, u):
    sums = torch.cumsum(w, 0)
    return min(int(torch.searchsorted(sums, u * sums[-1:], right=True)), int(torch.nonzero(w)[-1, 0]))


def _exact_verify(s):
    B, G, M = s["B"], s["G"], s["M"]
    T = s["temperature"].double().tolist() if isinstance(s["temperature"], torch.Tensor) else [s["temperature"]] * B
    drafts, u = s["drafts"].tolist(), s["uniforms"].double().tolist()
    tokens, accepted = [], []
    for b in range(B):
        out = []
        while True:
            i = len(out)
            w = _exact_weights(s["target"][b, i].double(), T[b])
            w /= w.sum()
            d = drafts[b][i] if i < G else -1
            if not 0 <= d < M:
                break
            if s["draft_logits"] is None or T[b] == 0:
                q = torch.zeros_like(w)
                q[d] = 1
            else:
                q = _exact_weights(s["draft_logits"][b, i].double(), T[b])
                q /= q.sum()
            if u[b][i] * float(q[d]) < float(w[d]):
                out.append(d)
                continue
            rest = torch.relu(w - q)
            if float(rest.sum()) > _LEAST_MASS:
                w = rest
            break
        accepted.append(len(out))
        out.append(_exact_pick(w, u[b][G]))
        tokens.append(out + [-1] * (G + 1 - len(out)))
    return torch.tensor(tokens, device="cuda"), torch.tensor(accepted, device="cuda", dtype=torch.int32)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "verify":
        return _exact_verify(s)
    if case["op"] == "sample":
        T = s["temperature"].double().tolist() if isinstance(s["temperature"], torch.Tensor) else [s["temperature"]] * case["N"]
        u = s["uniforms"].double().tolist()
        return torch.tensor([_exact_pick(_exact_weights(s["logits"][n].double(), T[n]), u[n]) for n in range(case["N"])], device="cuda")
    groups, E, k = case["groups"], case["E"], case["k"]
    x = s["logits"].double().requires_grad_()
    cols = s["cols"].long()
    real = (cols >= 0) & (cols < E)
    some = real.any(1)
    per = case["N"] // groups
    losses, zs, means, picks, rows = [], [], [], [], []
    for g in range(groups):
        part = slice(g * per, (g + 1) * per)
        mine = x[part][some[part]]
        n = max(1, mine.shape[0])
        count = torch.bincount(cols[part][real[part]], minlength=E)
        mean = torch.softmax(mine, 1).sum(0) / n
        losses.append(E * (count / max(1, int(count.sum())) * mean).sum())
        zs.append(torch.logsumexp(mine, 1).square().sum() / n)
        means.append(mean)
        picks.append(count)
        rows.append(mine.shape[0])
    losses, zs = torch.stack(losses), torch.stack(zs)
    if case["op"] == "balance":
        return (losses.detach(), zs.detach(), torch.stack(means).detach(), torch.stack(picks).to(torch.int32),
                torch.tensor(rows, device="cuda", dtype=torch.int32))
    all_of_it = (losses * s["grad_loss"].double()).sum() + (zs * s["grad_z"].double()).sum()
    if s["grad_picked"] is not None:
        at = torch.where(real, cols, 0)
        all_of_it = all_of_it + (torch.gather(x, 1, at) * s["grad_picked"].double() * real).sum()
    return torch.autograd.grad(all_of_it, x)[0]
