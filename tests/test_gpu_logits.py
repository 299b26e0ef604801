"""Log probabilities with entropy and top alternatives, distillation, and their gradients on the GPU against the definitions in 64 bits
(oracle/logits.py, numpy).

Tolerances, in units of 2^-24 (half a unit in the last place of an fp32 near 1), from the fp32 arithmetic that the definitions need:
  ln q = (x - m) / T - ln S.  Difference, 1 / T, product and the last subtraction round once each: 4 |x - m| / T, |ln q|.  Each term of S is
  off by three roundings of its exponent and one of exp2, an average of 12 such units for exponents that matter (entropies up to 12), and
  a sum of up to 512 terms in a row by a random walk of 512 roundings, 23: 64 for S in all, with ln S's own rounding 2 |ln S|.
  Entropy: 64 for each of S and A, of the size of 1 + ln S + |A / S T|.
  Gradients: q's relative error is that of exp(ln q), ln q from a rounded log-sum-exp; then the output's rounding.
Whole numbers (columns) are equal."""
import ctypes

import numpy as np
import pytest

from oracle import logits as definition

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}  # of a value with 24, 11, 8 significant bits, relative
TINY = {"f32": 2.0**-126, "f16": 2.0**-25, "bf16": 2.0**-126}
U = 2.0**-24


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_00822_amd as R

    R.load_library()
    return R


def wide(t):
    return t.detach().cpu().double().numpy()


def rows(N, M, dtype, seed, pad=0, shift=0, scale=3.0, mask=None):
    """Rows of logits as a view of a larger buffer of NaN: `pad` columns between rows, `shift` elements before the first."""
    gen = torch.Generator().manual_seed(seed)
    buf = torch.full((N * (M + pad) + shift + 64,), float("nan"), dtype=TYPES[dtype])
    x = buf[shift:shift + N * (M + pad)].view(N, M + pad)[:, :M]
    x.copy_((torch.randn((N, M), generator=gen) * scale - 2).to(TYPES[dtype]))
    if mask is not None:
        mask(x, gen)
    d = buf.cuda()
    return d[shift:shift + N * (M + pad)].view(N, M + pad)[:, :M], wide(x)


def near(got, want, tol, what):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    tol = np.broadcast_to(tol, want.shape)
    # a value beyond fp32 is its last finite number or infinite
    last = float(np.finfo(np.float32).max)
    same = (got == want) | (np.isnan(got) & np.isnan(want)) | ((np.abs(want) + tol >= last) & (np.sign(got) == np.sign(want)) & (np.abs(got) >= last * (1 - 2.0**-23)))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= tol)
    assert ok.all(), f"{what}: {np.argwhere(~ok)[:3].tolist()} got {got[~ok][:3]} want {want[~ok][:3]} tol {tol[~ok][:3]}"


def tol_logq(x, T, logq, lse):
    m = x.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        d = np.nan_to_num(np.abs(x - m), nan=0.0, posinf=0.0) / T
    ln_s = np.nan_to_num(lse - m[:, 0] / T, nan=0.0, posinf=0.0, neginf=0.0)
    return U * (4 * d + np.nan_to_num(np.abs(logq), posinf=0.0) + 2 * np.abs(ln_s)[:, None] + 64)


def check_forward(R, x, xh, tokens, k, T=1.0, got=None):
    N, M = xh.shape
    if got is None:
        got = R.rtopk_token_logprobs(x, tokens, k, T)
    th = tokens.cpu().numpy().reshape(N, -1)
    logq, lse = definition.log_softmax(xh, T)
    tol = tol_logq(xh, T, logq, lse)
    ok = (th >= 0) & (th < M)
    at = np.where(ok, th, 0)
    near(wide(got[0]).reshape(N, -1), definition.token_logprobs(xh, th, T), np.where(ok, np.take_along_axis(tol, at, 1), 0.0), "log probabilities")
    h = definition.entropy(logq)
    m = xh.max(axis=1)
    ln_s = np.nan_to_num(lse - m / T, nan=0.0, posinf=0.0, neginf=0.0)
    near(wide(got[1]), h, U * 64 * (1 + np.abs(ln_s) + np.abs(h - ln_s)), "entropy")
    near(wide(got[2]), lse, U * (64 + 2 * np.abs(ln_s) + 2 * np.nan_to_num(np.abs(lse), posinf=0.0) + 2 * np.nan_to_num(np.abs(m), posinf=0.0) / T), "log-sum-exp")
    assert len(got) == (5 if k else 3)
    if k:
        cols = definition.top(xh, k)
        assert np.array_equal(got[4].cpu().numpy(), cols), "columns of the alternatives"
        near(wide(got[3]), np.take_along_axis(logq, cols, 1), np.take_along_axis(tol, cols, 1), "alternatives")
    return got


def some_tokens(N, M, G, seed, dtype=torch.int64):
    gen = torch.Generator().manual_seed(seed)
    t = torch.randint(0, M, (N, G) if G else (N,), generator=gen)
    t.view(-1)[::7] = -100
    if t.numel() > 3:
        t.view(-1)[3] = M
    return t.to(dtype).cuda()


WIDTHS = [1, 2, 3, 7, 8, 9, 31, 63, 64, 65, 100, 255, 257, 1000, 1023, 2047, 2048, 2049, 4099, 8191, 16384, 32001, 50000]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", WIDTHS)
def test_forward_at_every_kind_of_width(dtype, M):
    R = _gpu()
    for N, T in ((1, 1.0), (3, 0.7), (37 if M <= 16384 else 9, 2.0)):
        x, xh = rows(N, M, dtype, seed=M + N, pad=N % 2 * 5, shift=N % 3)
        for k in sorted({0, 1, min(5, M), min(33, M), min(128, M)}):
            check_forward(R, x, xh, some_tokens(N, M, 0 if k % 2 else 3, seed=k), k, T)


@pytest.mark.parametrize("dtype,N,M,k", [("f32", 600, 5000, 20), ("bf16", 700, 5001, 20), ("f16", 1030, 2048, 32), ("bf16", 1030, 2048, 33), ("bf16", 520, 9001, 128),
                                         ("f32", 3, 262144, 20), ("bf16", 2, 262147, 128), ("f16", 1, 1000003, 64), ("f32", 1, 1 << 24, 5), ("bf16", 5, 131072, 0)])
def test_forward_of_many_rows_and_of_wide_ones(dtype, N, M, k):
    R = _gpu()
    x, xh = rows(N, M, dtype, seed=M)
    check_forward(R, x, xh, some_tokens(N, M, 0, 5, torch.int32), k)


def lowest(x, value, gen, keep):
    keep = torch.rand(x.shape, generator=gen) < keep
    x.masked_fill_(~keep, value)


MASKS = {
    "a tail of -inf": lambda x, g: x[:, -(x.shape[1] // 3):].fill_(float("-inf")),
    "few columns left": lambda x, g: lowest(x, float("-inf"), g, 0.002),
    "none left": lambda x, g: x[::2].fill_(float("-inf")),
    "one left": lambda x, g: (x.fill_(float("-inf")), x[:, x.shape[1] * 2 // 3].fill_(1.5)),
    "the type's lowest value": lambda x, g: lowest(x, torch.finfo(x.dtype).min, g, 0.01),
    "all equal": lambda x, g: x.fill_(0.25),
    "all the type's lowest value": lambda x, g: x.fill_(torch.finfo(x.dtype).min),
    "four levels": lambda x, g: x.copy_(torch.randint(0, 4, x.shape, generator=g).to(x.dtype)),
    "zeros of both signs": lambda x, g: x.copy_(torch.where(torch.rand(x.shape, generator=g) < 0.5, -0.0, 0.0).to(x.dtype)),
    "one far above": lambda x, g: x[:, 1].fill_(60.0),
    "ascending": lambda x, g: x.copy_((torch.arange(x.shape[1]) / x.shape[1]).expand(x.shape).to(x.dtype)),
    "descending": lambda x, g: x.copy_((-torch.arange(x.shape[1]) / x.shape[1]).expand(x.shape).to(x.dtype)),
    "the largest where one thread reads": lambda x, g: x.copy_(torch.where(torch.arange(x.shape[1]) % 2048 < 8, 5.0 + torch.rand(x.shape, generator=g), x.float()).to(x.dtype)),
    "the largest where a few threads read": lambda x, g: x.copy_(torch.where(torch.arange(x.shape[1]) % 8192 < 40, 5.0 + torch.rand(x.shape, generator=g), x.float()).to(x.dtype)),
    "a plateau at the end": lambda x, g: x[:, -x.shape[1] // 4:].fill_(30.0),
}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mask", list(MASKS))
@pytest.mark.parametrize("N,M", [(3, 40000), (2, 2000), (520, 3000)])
def test_forward_under_masks_ties_and_crowds(mask, dtype, N, M):
    R = _gpu()
    x, xh = rows(N, M, dtype, seed=N + M, mask=MASKS[mask])
    for k in (0, 1, 20, 128):
        check_forward(R, x, xh, some_tokens(N, M, 2, k), k)
        check_forward(R, x, xh, some_tokens(N, M, 2, k), k, got=whole(R, x, some_tokens(N, M, 2, k), k))


def whole(R, x, tokens, k, T=1.0):
    """The call without scratch memory: a workgroup for each row."""
    N, M = x.shape
    G = tokens.shape[1]
    out = [torch.full(s, 7.5, device="cuda") for s in ((N, G), (N,), (N,), (N, k))] + [torch.full((N, k), -7, dtype=torch.int32, device="cuda")]
    dtype = [torch.float32, torch.float16, torch.bfloat16].index(x.dtype)
    stream = torch.cuda.current_stream().cuda_stream
    rc = R.load_library().rtopk_token_logprobs(x.data_ptr(), dtype, N, M, x.stride(0), tokens.data_ptr(), tokens.element_size(), G, k, T, out[0].data_ptr(),
                                               out[1].data_ptr(), out[2].data_ptr(), out[3].data_ptr(), out[4].data_ptr(), None, 0, stream)
    assert rc == 0
    return out if k else out[:3]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,k,spread", [(131072, 20, 8192), (131072, 128, 8192), (262144, 100, 2048)])
def test_more_columns_reach_the_floor_than_are_listed(dtype, M, k, spread):
    """The largest columns are all read by few threads, thousands of them: every layout's second search."""
    R = _gpu()
    crowd = lambda x, g: x.copy_(torch.where(torch.arange(M) % spread < 64, 20 + 4 * torch.rand(x.shape, generator=g), x.float()).to(x.dtype))  # noqa: E731
    x, xh = rows(2, M, dtype, seed=M + k, mask=crowd)
    t = some_tokens(2, M, 1, 3)
    check_forward(R, x, xh, t, k)
    check_forward(R, x, xh, t, k, got=whole(R, x, t, k))
    many = x[:1].expand(600, M).contiguous()  # a workgroup of four wavefronts for each row
    got = R.rtopk_token_logprobs(many, t[:1].expand(600, 1).contiguous(), k)
    check_forward(R, x[:1], xh[:1], t[:1], k, got=[g[:1] for g in got])
    for g in got:
        assert (g == g[:1]).all(), "equal rows, equal results"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", ["nan", "inf"])
@pytest.mark.parametrize("M", [100, 5000, 70000])
def test_a_row_that_is_not_a_number_spoils_itself_only(dtype, bad, M):
    R = _gpu()
    N, k = 6, 20

    def spoil(x, g):
        x[1, M // 2] = float(bad)
        x[3] = float(bad)
        x[4, ::3] = float(bad)

    x, xh = rows(N, M, dtype, seed=M, mask=spoil)
    t = torch.full((N,), M // 3, dtype=torch.int64, device="cuda")
    good = [0, 2, 5]
    got = R.rtopk_token_logprobs(x, t, k)
    check_forward(R, x[good], xh[good], t[good], k, got=[g[good] for g in got])
    for n in (1, 3, 4):
        assert torch.isnan(got[0][n]) and torch.isnan(got[1][n]) and torch.isnan(got[2][n])
        cols = got[4][n].cpu().numpy()
        assert len(set(cols.tolist())) == k and cols.min() >= 0 and cols.max() < M
    dx = wide(R.rtopk_token_logprobs_backward(torch.ones(N, device="cuda"), x, t, got[2], grad_entropy=torch.ones(N, device="cuda"), entropy=got[1]))
    assert np.isfinite(dx[good]).all() and np.isnan(dx[[1, 3, 4]]).any(axis=1).all()
    # a row that is left out is not looked at
    t[1], t[3], t[4] = -100, -100, M
    dx = wide(R.rtopk_token_logprobs_backward(torch.ones(N, device="cuda"), x, t, got[2]))
    assert (dx[[1, 3, 4]] == 0).all() and (dx[good] != 0).any()


# ---- gradients ----

def tol_q(xh, T, lse):
    """Of q relative to itself.  Beyond a log-sum-exp of 1024 the row's sums are taken again, and q is as exact as in the forward pass."""
    top = xh.max(axis=1, keepdims=True)
    ln_s = np.nan_to_num(lse[:, None] - top / T, nan=0.0, posinf=0.0, neginf=0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        again = U * (64 + 4 * np.nan_to_num(np.abs(xh - top), nan=0.0, posinf=0.0) / T + 2 * np.abs(ln_s))
    far = ~(np.abs(lse)[:, None] <= 1024)
    return np.where(far, again, tol_q_saved(xh, T, lse))


def tol_q_saved(xh, T, lse):
    with np.errstate(invalid="ignore"):
        return U * (64 + 4 * np.nan_to_num(np.abs(xh), posinf=0.0) / T + 4 * np.nan_to_num(np.abs(lse), posinf=0.0)[:, None])


def check_token_gradient(R, x, xh, tokens, T, entropy, seed, dtype, out=None):
    N, M = xh.shape
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(tokens.shape, generator=gen).cuda()
    ge = torch.randn((N,), generator=gen).cuda() if entropy else None
    _, h, lse = R.rtopk_token_logprobs(x, tokens, 0, T)
    dx = R.rtopk_token_logprobs_backward(g, x, tokens, lse, T, grad_entropy=ge, entropy=h if entropy else None, grad_logits=out)
    assert dx.dtype == x.dtype and tuple(dx.shape) == (N, M)
    th, gh = tokens.cpu().numpy().reshape(N, -1), wide(g).reshape(N, -1)
    want = definition.token_gradient(xh, th, gh, wide(ge) if entropy else None, T)
    logq, lse_h = definition.log_softmax(xh, T)
    q = np.exp(logq)
    ok = (th >= 0) & (th < M)
    size = np.abs(gh * ok).sum(1, keepdims=True) * q
    if entropy:
        size = size + np.abs(wide(ge))[:, None] * q * (np.abs(np.where(q == 0, 0, logq)) + definition.entropy(logq)[:, None] + 1)
    at_tokens = np.zeros_like(want)
    np.add.at(at_tokens, (np.arange(N)[:, None], np.where(ok, th, 0)), np.abs(gh * ok))
    tol = (tol_q(xh, T, lse_h) * size + 8 * U * at_tokens) / T + HALF_ULP[dtype] * np.abs(want) * 1.01 + TINY[dtype]
    near(wide(dx), want, tol, "gradient")
    return dx


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", [1, 2, 7, 9, 64, 100, 1000, 2049, 4099, 8192, 16385, 50001])
def test_token_gradient(dtype, M):
    R = _gpu()
    for N, T, G, entropy in ((1, 1.0, 0, False), (5, 0.7, 0, True), (34, 2.0, 3, True), (9, 1.0, 70, False)):
        x, xh = rows(N, M, dtype, seed=M + N, pad=G, shift=N % 3)
        check_token_gradient(R, x, xh, some_tokens(N, M, G, seed=N), T, entropy, N, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mask", ["a tail of -inf", "few columns left", "none left", "one left", "the type's lowest value", "all the type's lowest value", "all equal", "one far above"])
def test_token_gradient_under_masks(mask, dtype):
    R = _gpu()
    for N, M in ((4, 3000), (3, 40001)):
        x, xh = rows(N, M, dtype, seed=M, mask=MASKS[mask])
        tokens = torch.full((N, 1), M * 2 // 3, device="cuda", dtype=torch.int32)
        for entropy in (False, True):
            check_token_gradient(R, x, xh, tokens, 1.0, entropy, 3, dtype)
            check_token_gradient(R, x.clone(), xh, tokens, 1.0, entropy, 3, dtype)


def teacher_list(N, M, k, seed, tdtype="f32", log_probs=False, sort=True, spoil=True):
    gen = torch.Generator().manual_seed(seed)
    vals = (torch.randn((N, k), generator=gen) * 2 + 3)
    if log_probs:
        vals = torch.log_softmax(vals, 1) - 0.1
    cols = torch.stack([torch.randperm(M, generator=gen)[:k] if k <= M else torch.randint(0, M, (k,), generator=gen) for _ in range(N)])
    if sort:
        cols = cols.sort(1)[0]
    if spoil and k > 2:
        cols[::2, 1] = -1
        cols[::3, 0] = M
        vals[::4, 2] = float("-inf")
    if spoil and N > 4:
        cols[4] = -1  # a row without entries
    vals = vals.to(TYPES[tdtype])
    return vals.cuda(), cols.to(torch.int32).cuda(), wide(vals), cols.numpy()


def tol_distill(xh, vh, ch, T, log_probs):
    """(tolerance of the loss, p, log q at the list)"""
    M = xh.shape[1]
    p, lp, at = definition.teacher(vh, ch, M, T, log_probs)
    logq, lse = definition.log_softmax(xh, T)
    lq = np.take_along_axis(logq, at, 1)
    t = np.take_along_axis(tol_logq(xh, T, logq, lse), at, 1)
    spread = np.abs(np.where(np.isfinite(vh), vh, 0)).max(axis=1, keepdims=True) / T
    # ln p: as ln q, over the list; p's own relative error is ln p's; the sum of k products
    t_lp = U * (8 * spread + 2 * np.abs(lp) + 64)
    with np.errstate(invalid="ignore"):
        term = np.abs(np.where(p > 0, lp - lq, 0.0))
    term = np.where(np.isfinite(term), term, 0.0)
    return (p * (t + t_lp + t_lp * term + 8 * U * term)).sum(axis=1), p, t_lp


def check_distill(R, x, xh, lists, T, log_probs, dtype, seed, in_place=False, weights=None):
    vals, cols, vh, ch = lists
    N, M = xh.shape
    want = definition.distill(xh, vh, ch, T, log_probs)
    tol, p, t_lp = tol_distill(xh, vh, ch, T, log_probs)
    loss, lse = R.rtopk_distill(x, vals, cols, T, log_probs=log_probs)
    near(wide(loss), want, tol, "loss")
    _, lse_h = definition.log_softmax(xh, T)
    m = np.nan_to_num(np.abs(xh.max(axis=1)), posinf=0.0) / T
    near(wide(lse), lse_h, U * (64 + 4 * np.nan_to_num(np.abs(lse_h), posinf=0.0) + 4 * m), "log-sum-exp")
    if weights is None:
        weights = torch.randn((N,), generator=torch.Generator().manual_seed(seed)).cuda()
    wh = wide(weights)
    dwant = definition.distill_gradient(xh, vh, ch, wh, T, log_probs)
    q = np.exp(definition.log_softmax(xh, T)[0])
    at_list = np.zeros_like(dwant)
    np.add.at(at_list, (np.arange(N)[:, None], np.where((ch >= 0) & (ch < M), ch, 0)), p * (t_lp + 8 * U))
    dtol = np.abs(wh)[:, None] / T * (tol_q(xh, T, lse_h) * q * p.sum(1, keepdims=True) + q * (p * t_lp).sum(1, keepdims=True) + at_list)
    dtol = dtol + HALF_ULP[dtype] * np.abs(dwant) * 1.01 + TINY[dtype]
    dx = R.rtopk_distill_backward(weights, x, vals, cols, lse, T, log_probs=log_probs)
    near(wide(dx), dwant, dtol, "gradient from the saved log-sum-exp")
    loss2, dx = R.rtopk_distill_with_grad(weights, x, vals, cols, T, log_probs=log_probs, grad_logits=x if in_place else None)
    assert dx.dtype == x.dtype
    near(wide(loss2), want, tol, "loss, with gradient")
    near(wide(dx), dwant, dtol, "gradient")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,k", [(1, 1), (2, 2), (9, 4), (64, 64), (100, 7), (1000, 1), (1000, 1000), (2048, 16), (2049, 100), (4099, 1024), (8192, 64), (16385, 33), (50001, 128)])
def test_distillation(dtype, M, k):
    R = _gpu()
    for n, (N, T, log_probs, tdtype) in enumerate(((1, 1.0, False, "f32"), (7, 0.7, True, "f32"), (33 if M < 16000 else 6, 2.0, False, "bf16"), (5, 1.0, False, "f16"))):
        x, xh = rows(N, M, dtype, seed=M + N, pad=n, shift=n % 3)
        check_distill(R, x, xh, teacher_list(N, M, k, N + k, tdtype, log_probs, sort=n % 2 == 0), T, log_probs, dtype, N, in_place=n == 2)


@pytest.mark.parametrize("dtype,N,M,k", [("f32", 600, 3000, 32), ("bf16", 700, 5001, 20), ("f16", 1030, 2048, 128), ("bf16", 520, 9001, 400), ("bf16", 2, 262147, 64)])
def test_distillation_of_many_rows_and_of_wide_ones(dtype, N, M, k):
    R = _gpu()
    x, xh = rows(N, M, dtype, seed=M)
    check_distill(R, x, xh, teacher_list(N, M, k, N), 1.0, False, dtype, N, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_columns_that_come_twice_add_up(dtype):
    R = _gpu()
    for N, M, k in ((5, 40, 64), (3, 5000, 300), (600, 300, 400)):
        x, xh = rows(N, M, dtype, seed=N)
        vals, cols, vh, _ = teacher_list(N, M, k, 5, spoil=False)
        cols = torch.randint(0, min(M, 50), (N, k), generator=torch.Generator().manual_seed(1)).to(torch.int32)
        check_distill(R, x, xh, (vals, cols.cuda(), vh, cols.numpy().astype(np.int64)), 1.0, False, dtype, 3)
        check_distill(R, x, xh, (vals, cols.sort(1)[0].cuda(), vh, cols.sort(1)[0].numpy().astype(np.int64)), 1.0, False, dtype, 3)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mask", ["a tail of -inf", "few columns left", "none left", "one left", "all equal", "one far above"])
def test_distillation_under_masks(mask, dtype):
    """A masked column on the teacher's list makes the loss infinite; the gradient stays finite, and a row of nothing but -inf has none."""
    R = _gpu()
    for N, M, k in ((4, 3000, 30), (3, 40001, 30), (530, 2100, 30)):
        x, xh = rows(N, M, dtype, seed=M, mask=MASKS[mask])
        check_distill(R, x, xh, teacher_list(N, M, k, M), 1.0, False, dtype, 3)


def test_a_teacher_without_entries_makes_a_row_that_is_not_looked_at():
    R = _gpu()
    for N, M in ((5, 3000), (5, 60000), (600, 2500)):
        x, _ = rows(N, M, "bf16", seed=1, mask=lambda x, g: x.fill_(float("nan")))
        vals, cols = torch.zeros((N, 4), device="cuda"), torch.full((N, 4), -1, dtype=torch.int32, device="cuda")
        w = torch.ones(N, device="cuda")
        loss, dx = R.rtopk_distill_with_grad(w, x, vals, cols)
        assert (loss == 0).all() and (dx == 0).all()
        loss, lse = R.rtopk_distill(x, vals, cols)
        assert (loss == 0).all()
        assert (R.rtopk_distill_backward(w, x, vals, cols, lse) == 0).all()


def test_gradients_against_differences():
    """The kernels' gradients against central differences of the definitions in 64 bits: h = 2^-12, off by h^2 / 6 of the third derivative
    (below 4 for these sizes) and by 2^-52 |value| / h."""
    R = _gpu()
    N, M, T = 3, 50, 0.8
    x, xh = rows(N, M, "f32", seed=3, scale=1.0)
    tokens = torch.tensor([[3, 7], [49, 49], [-1, 0]]).cuda()
    g, ge = torch.randn((N, 2), generator=torch.Generator().manual_seed(1)), torch.randn((N,), generator=torch.Generator().manual_seed(2))
    vals, cols, vh, ch = teacher_list(N, M, 8, 4, spoil=False)
    w = torch.randn((N,), generator=torch.Generator().manual_seed(6))

    def policy(v):
        logq, _ = definition.log_softmax(v, T)
        return (definition.token_logprobs(v, tokens.cpu().numpy(), T) * g.double().numpy()).sum() + (definition.entropy(logq) * ge.double().numpy()).sum()

    def distilled(v):
        return (definition.distill(v, vh, ch, T) * w.double().numpy()).sum()

    _, h, lse = R.rtopk_token_logprobs(x, tokens, 0, T)
    d1 = wide(R.rtopk_token_logprobs_backward(g.cuda(), x, tokens, lse, T, grad_entropy=ge.cuda(), entropy=h))
    d2 = wide(R.rtopk_distill_with_grad(w.cuda(), x, vals, cols, T)[1])
    e = 2.0**-12
    for f, d in ((policy, d1), (distilled, d2)):
        for n, v in [(0, 3), (0, 7), (0, 11), (1, 49), (1, 0), (2, 0), (2, 1), (0, int(ch[0, 2])), (2, int(ch[2, 7]))]:
            up, down = xh.copy(), xh.copy()
            up[n, v] += e
            down[n, v] -= e
            assert abs(d[n, v] - (f(up) - f(down)) / (2 * e)) < e * e / 6 * 4 * 4 + 1e-10 + 200 * U, (n, v)


# ---- memory, streams, graphs ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,M", [(7, 1001), (3, 40003), (600, 2307)])
def test_outputs_of_the_caller_are_written_inside_only(dtype, N, M):
    R = _gpu()
    k, pad, item = 5, 3, TYPES[dtype]
    x, xh = rows(N, M, dtype, seed=M)
    t = some_tokens(N, M, 2, 1)

    def guarded(shape, dt):
        n = int(np.prod(shape))
        buf = torch.full((n + 128,), 7, dtype=dt, device="cuda")
        return buf, buf[64:64 + n].view(shape)

    made = [guarded(s, d) for s, d in (((N, 2), torch.float32), ((N,), torch.float32), ((N,), torch.float32), ((N, k), torch.float32), ((N, k), torch.int32))]
    got = R.rtopk_token_logprobs(x, t, k, 1.0, *[v for _, v in made])
    assert all(a is v for a, (_, v) in zip(got, made))
    check_forward(R, x, xh, t, k, got=got)
    vals, cols, _, _ = teacher_list(N, M, 9, 2)
    buf = torch.full((N * (M + pad) + 64,), 7, dtype=item, device="cuda")
    dx = buf[31:31 + N * (M + pad)].view(N, M + pad)[:, :M]
    w = torch.ones(N, device="cuda")
    want = R.rtopk_distill_with_grad(w, x, vals, cols)[1]
    assert R.rtopk_distill_with_grad(w, x, vals, cols, grad_logits=dx)[1] is dx
    torch.testing.assert_close(dx, want, rtol=0, atol=0)
    around = buf[31:31 + N * (M + pad)].view(N, M + pad)[:, M:]
    assert (buf[:31] == 7).all() and (buf[31 + N * (M + pad):] == 7).all() and (around == 7).all()
    for b, v in made:
        assert (b[:64] == 7).all() and (b[-64:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,M", [(3, 40001), (600, 2307)])
def test_a_gradient_in_its_logits_place(dtype, N, M):
    R = _gpu()
    x, xh = rows(N, M, dtype, seed=M, pad=5)
    t = some_tokens(N, M, 3, 1)
    _, h, lse = R.rtopk_token_logprobs(x, t)
    g, ge = torch.randn((N, 3), device="cuda"), torch.randn((N,), device="cuda")
    want = R.rtopk_token_logprobs_backward(g, x, t, lse, grad_entropy=ge, entropy=h)
    vals, cols, _, _ = teacher_list(N, M, 40, 2, sort=False)
    loss, want2 = R.rtopk_distill_with_grad(ge, x, vals, cols)
    lse2 = R.rtopk_distill(x, vals, cols)[1]
    want3 = R.rtopk_distill_backward(ge, x, vals, cols, lse2)
    keep = torch.as_strided(x, x.shape, x.stride(), x.storage_offset()).clone()
    assert torch.equal(R.rtopk_token_logprobs_backward(g, x, t, lse, grad_entropy=ge, entropy=h, grad_logits=x), want)
    x.copy_(keep)
    loss2, _ = R.rtopk_distill_with_grad(ge, x, vals, cols, grad_logits=x)
    assert torch.equal(x, want2) and torch.equal(loss, loss2)
    x.copy_(keep)
    R.rtopk_distill_backward(ge, x, vals, cols, lse2, grad_logits=x)
    assert torch.equal(x, want3)


def test_elements_beyond_32_bits():
    R = _gpu()
    N, M = 17000, 131072 + 8  # 4.4 GB, offsets beyond 2^31 elements
    x = torch.full((N, M), -20.0, dtype=torch.bfloat16, device="cuda")
    last = torch.arange(N - 3, N, device="cuda")
    x[last] = (torch.randn((3, M), generator=torch.Generator().manual_seed(1)) * 3).to(torch.bfloat16).cuda()
    t = torch.full((N,), 77, device="cuda")
    got = R.rtopk_token_logprobs(x, t, 4)
    xh = wide(x[last])
    check_forward(R, x[last], xh, t[last], 4, got=[g[last] for g in got])
    dx = R.rtopk_token_logprobs_backward(torch.ones(N, device="cuda"), x, t, got[2])
    want = definition.token_gradient(xh, np.full((3, 1), 77), np.ones((3, 1)))
    _, lse = definition.log_softmax(xh)
    near(wide(dx[last]), want, tol_q(xh, 1.0, lse) * np.abs(want) + 8 * U + HALF_ULP["bf16"] * 1.01 * np.abs(want), "gradient")
    cols, vals = torch.arange(5, device="cuda", dtype=torch.int32).expand(N, 5).contiguous(), torch.ones((N, 5), device="cuda")
    loss, dx = R.rtopk_distill_with_grad(torch.ones(N, device="cuda"), x, vals, cols, grad_logits=dx)
    vh, ch = np.ones((3, 5)), np.tile(np.arange(5), (3, 1))
    near(wide(loss[last]), definition.distill(xh, vh, ch), tol_distill(xh, vh, ch, 1.0, False)[0], "loss")
    want = definition.distill_gradient(xh, vh, ch, np.ones(3))
    near(wide(dx[last]), want, tol_q(xh, 1.0, lse) * np.abs(want) + 64 * U + HALF_ULP["bf16"] * 1.01 * np.abs(want), "gradient")


@pytest.mark.parametrize("N,M", [(2, 60000), (600, 3000)])
def test_streams_and_graphs(N, M):
    """Work goes to the current stream; a captured call gives the eager results at every replay, with other work between."""
    R = _gpu()
    x, _ = rows(N, M, "bf16", seed=1)
    x = x.contiguous()
    t = some_tokens(N, M, 0, 1)
    vals, cols, _, _ = teacher_list(N, M, 16, 2)
    w = torch.rand(N, device="cuda")

    def calls():
        lp, h, lse, tl, tc = R.rtopk_token_logprobs(x, t, 7)
        d = R.rtopk_token_logprobs_backward(w, x, t, lse, grad_entropy=w, entropy=h)
        loss, lse2 = R.rtopk_distill(x, vals, cols)
        return [lp, h, lse, tl, tc, d, loss, lse2, R.rtopk_distill_backward(w, x, vals, cols, lse2), *R.rtopk_distill_with_grad(w, x, vals, cols)]

    want = [o.clone() for o in calls()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    keep = x.clone()
    for turn in range(4):
        x.copy_(keep.roll(turn, 1))
        expect = [o.clone() for o in calls()]
        for o in out:
            o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, expect)), turn
        (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()


def test_repeated_calls_give_the_same_bits():
    R = _gpu()
    for N, M in ((2, 100000), (700, 3000)):
        x, _ = rows(N, M, "f32", seed=5)
        t = some_tokens(N, M, 0, 1)
        vals, cols, _, _ = teacher_list(N, M, 300, 2)
        w = torch.rand(N, device="cuda")
        first = [*R.rtopk_token_logprobs(x, t, 128), *R.rtopk_distill_with_grad(w, x, vals, cols)]
        for _ in range(5):
            again = [*R.rtopk_token_logprobs(x, t, 128), *R.rtopk_distill_with_grad(w, x, vals, cols)]
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_no_rows_and_no_tokens():
    R = _gpu()
    x = torch.empty((0, 100), device="cuda")
    got = R.rtopk_token_logprobs(x, torch.empty((0,), dtype=torch.int64, device="cuda"), 5)
    assert [tuple(g.shape) for g in got] == [(0,), (0,), (0,), (0, 5), (0, 5)]
    x, xh = rows(3, 1000, "f32", seed=1)
    none = torch.empty((3, 0), dtype=torch.int64, device="cuda")
    _, h, lse = check_forward(R, x, xh, none, 0)
    ge = torch.ones(3, device="cuda")
    dx = wide(R.rtopk_token_logprobs_backward(torch.empty((3, 0), device="cuda"), x, none, lse, grad_entropy=ge, entropy=h))
    want = definition.token_gradient(xh, np.empty((3, 0), dtype=np.int64), np.empty((3, 0)), np.ones(3))
    q = np.exp(definition.log_softmax(xh)[0])
    near(dx, want, tol_q(xh, 1.0, wide(lse)) * q * 30 + 2**-24 * np.abs(want), "entropy's gradient")


def test_the_selections_pairs_are_a_teachers_list():
    """rtopk_rowwise_exact on the teacher's logits, and rtopk_token_logprobs on them, feed the student's loss."""
    R = _gpu()
    N, M, k, T = 40, 5000, 24, 1.0
    teacher, th = rows(N, M, "f32", seed=1)
    x, xh = rows(N, M, "bf16", seed=2)
    vals, cols = R.rtopk_rowwise_exact(teacher.contiguous(), k)
    check_distill(R, x, xh, (vals, cols, wide(vals), cols.cpu().numpy().astype(np.int64)), T, False, "bf16", 1)
    top, topc = R.rtopk_token_logprobs(teacher, torch.zeros(N, dtype=torch.int64, device="cuda"), k, T)[3:]
    check_distill(R, x, xh, (top, topc, wide(top), topc.cpu().numpy().astype(np.int64)), T, True, "bf16", 1)
    assert np.array_equal(np.sort(topc.cpu().numpy(), 1), cols.cpu().numpy())


def test_refusals():
    R = _gpu()
    x = torch.zeros((4, 100), device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    v, c, w = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 8), dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda")
    lse = torch.ones(4, device="cuda")
    line = torch.zeros(1000, device="cuda")
    for bad in (lambda: R.rtopk_token_logprobs(x.double(), t), lambda: R.rtopk_token_logprobs(x.cpu(), t), lambda: R.rtopk_token_logprobs(x.t(), t),
                lambda: R.rtopk_token_logprobs(x[:1].expand(4, 100), t), lambda: R.rtopk_token_logprobs(x, t[:3]), lambda: R.rtopk_token_logprobs(x, t.float()),
                lambda: R.rtopk_token_logprobs(x, t.cpu()), lambda: R.rtopk_token_logprobs(x, t, 3, out_top_cols=torch.zeros((4, 3), device="cuda")),
                lambda: R.rtopk_token_logprobs(x, t, 0, out_top_cols=c), lambda: R.rtopk_token_logprobs_backward(w[:2], x, t, lse),
                lambda: R.rtopk_token_logprobs_backward(w, x, t, lse, grad_entropy=w), lambda: R.rtopk_token_logprobs_backward(w, x, t, lse.double()),
                lambda: R.rtopk_token_logprobs_backward(w, x, t, lse, grad_logits=x.half()), lambda: R.rtopk_distill(x, v, c.long()),
                lambda: R.rtopk_distill(x, v, c[:, :4]), lambda: R.rtopk_distill(x, v.double(), c), lambda: R.rtopk_distill(x, v[:3], c[:3]),
                lambda: R.rtopk_distill_with_grad(w.double(), x, v, c), lambda: R.rtopk_distill_with_grad(w, x, v, c, grad_logits=x[:, :50])):
        with pytest.raises(ValueError):
            bad()
    for status, bad in ((-2, lambda: R.rtopk_token_logprobs(x, t, 101)), (-2, lambda: R.rtopk_token_logprobs(torch.zeros((4, 500), device="cuda"), t, 129)),
                        (-2, lambda: R.rtopk_token_logprobs(x, t, -1)), (-9, lambda: R.rtopk_token_logprobs(x, t, 0, 0.0)),
                        (-9, lambda: R.rtopk_token_logprobs(x, t, 0, -1.0)), (-9, lambda: R.rtopk_token_logprobs(x, t, 0, float("nan"))),
                        (-9, lambda: R.rtopk_distill(x, v, c, float("inf"))), (-9, lambda: R.rtopk_distill(x, v, c, 1e-42)),
                        (-2, lambda: R.rtopk_token_logprobs(x, torch.zeros((4, 1025), dtype=torch.int64, device="cuda"))),
                        (-2, lambda: R.rtopk_distill(x, torch.zeros((4, 1025), device="cuda"), torch.zeros((4, 1025), dtype=torch.int32, device="cuda"))),
                        (-8, lambda: R.rtopk_distill_with_grad(w, x, v, c, out_loss=w)), (-8, lambda: R.rtopk_token_logprobs(x, t, out_lse=lse, out_entropy=lse)),
                        (-8, lambda: R.rtopk_distill_backward(w, line[:400].view(4, 100), v, c, lse, grad_logits=line[100:500].view(4, 100)))):
        with pytest.raises(R.RTopKError) as e:
            bad()
        assert e.value.status == status


def test_c_call_with_optional_outputs_left_out():
    R = _gpu()
    x, xh = rows(5, 3000, "f16", seed=1)
    t = some_tokens(5, 3000, 1, 1, torch.int32)
    out = torch.full((5, 1), 7.5, device="cuda")
    vp = ctypes.c_void_p
    rc = R.load_library().rtopk_token_logprobs(vp(x.data_ptr()), 1, 5, 3000, x.stride(0), vp(t.data_ptr()), 4, 1, 0, 1.0, vp(out.data_ptr()), None, None, None, None,
                                               None, 0, vp(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    logq, lse = definition.log_softmax(xh)
    th = t.cpu().numpy()
    near(wide(out), definition.token_logprobs(xh, th), tol_logq(xh, 1.0, logq, lse).max(axis=1, keepdims=True), "log probabilities")
