"""A router's balance loss and its gradient on the GPU against their definitions in 64 bits (oracle/balance.py, numpy).

Tolerances, in units of U = 2^-24.  A probability: its exponent (x - m) log2(e) is off by two roundings of itself, 2 D for D = max |x - m|, exp2 by 2, the sum
over E and the division by 12 more: (2 D + 14) of its value.  Sums over tokens run over 64 of them in fp32, 64 roundings at most, and in 64 bits beyond;
then an output's own rounding.  A log-sum-exp: D U of exponents weighed by their probabilities, ln's rounding and the last sum's: (2 D + 16 + 2 |lse|).
Gradients: p (w + 2 g_z lse / n - sum p w): p's error and 8 roundings, of the size of the terms; then half a step of the type.  Counts are equal."""
import numpy as np
import pytest

from oracle import balance as definition

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0**-24
TINY = {"f32": 2.0**-126, "f16": 2.0**-25, "bf16": 2.0**-126}


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_00822_amd as R

    R.load_library()
    return R


def wide(t):
    return t.detach().cpu().double().numpy()


def inputs(N, E, k, dtype, seed, pad=0, shift=0, ignored=0, bytes=4, scale=2.0):
    gen = torch.Generator().manual_seed(seed)
    buf = torch.full((N * (E + pad) + shift + 64,), float("nan"), dtype=TYPES[dtype])
    x = buf[shift:shift + N * (E + pad)].view(N, E + pad)[:, :E]
    x.copy_((torch.randn((N, E), generator=gen) * scale + torch.randn((E,), generator=gen)).to(TYPES[dtype]))
    cols = torch.topk(x.float(), k, dim=1)[1].sort(dim=1)[0] if N else torch.zeros((0, k), dtype=torch.int64)
    if ignored:
        cols[ignored - 1::ignored] = -1
    cols = cols.to(torch.uint8) if bytes == 1 else cols.to(torch.int32)
    d = buf.cuda()
    return d[shift:shift + N * (E + pad)].view(N, E + pad)[:, :E], cols.cuda()


def errors(x, keep=None):
    """D of each row, its log-sum-exp and the bound of its error."""
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(1, keepdims=True)
        d = np.where(np.isfinite(x), np.abs(x - m), 0.0)
        D = np.minimum(np.nan_to_num(d).max(1), 110.0)  # beyond, a probability is 0
        p, lse = definition._softmax(x)
    return D, p, lse, U * (2 * D + 16 + 2 * np.abs(np.nan_to_num(lse, posinf=0, neginf=0)))


def near(got, want, tol, what):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    ok = (np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), f"{what}: {np.argwhere(~ok)[:3].tolist()} got {got[~ok][:3]} want {want[~ok][:3]} tol {np.broadcast_to(tol, want.shape)[~ok][:3]}"


def check_forward(R, x, cols, groups=1, got=None):
    got = R.rtopk_balance_loss(x, cols, groups) if got is None else got
    xh, ch = wide(x), cols.cpu().numpy().astype(np.int64)
    loss, z, probs, counts, rows = definition.loss(xh, ch, groups)
    assert got[3].cpu().numpy().tolist() == counts.tolist() and got[4].cpu().numpy().tolist() == rows.tolist()
    if xh.shape[0] == 0:
        D, e_z = 0.0, 0.0
    else:
        D, _, lse, e = errors(xh)
        D = D.max()
        finite = np.nan_to_num(lse, posinf=0, neginf=0)
        e_z = (2 * np.abs(finite) * e).max() + 66 * U * z
    rel = U * (2 * D + 14 + 64 + 1)
    near(wide(got[2]), probs, rel * probs + TINY["f32"], "probs")
    near(wide(got[0]), loss, (rel + U) * loss, "loss")
    with np.errstate(over="ignore"):
        near(wide(got[1]), z.astype(np.float32), np.where(z < 3.4e38, e_z, 0.0), "z")  # (beyond fp32: infinite)
    return got


def check_gradient(R, x, cols, counts, rows, grad_loss, grad_z=None, grad_vals=None, before=None, **more):
    xh, ch = wide(x if before is None else before), cols.cpu().numpy().astype(np.int64)
    got = R.rtopk_balance_loss_backward(grad_loss, x, cols, counts, rows, grad_z, grad_vals, **more)
    c, n = counts.cpu().numpy().astype(np.int64), rows.cpu().numpy().astype(np.int64)
    gl, gz, gv = wide(grad_loss), wide(grad_z) if grad_z is not None else None, wide(grad_vals) if grad_vals is not None else None
    want = definition.gradient(xh, ch, c, n, gl, gz, gv)
    D, p, lse, e_lse = errors(xh)
    N, E = xh.shape
    g = np.arange(N) // (N // c.shape[0])
    over = 1 / np.maximum(1, n)[g]
    w = E * np.abs(gl[g])[:, None] * c[g] / np.maximum(1, c.sum(1))[g][:, None] * over[:, None]
    zf = 2 * np.abs(gz[g]) * over if gz is not None else np.zeros(N)
    lse_f = np.abs(np.nan_to_num(lse, posinf=0, neginf=0))
    size = w + np.nan_to_num(p * w).sum(1)[:, None] + (zf * lse_f)[:, None]
    tol = p * (U * (2 * D[:, None] * 2 + 36) * size + (zf * e_lse)[:, None])
    near_type = torch.finfo(x.dtype).eps / 2
    if gv is not None:  # sums of the picked values' gradients in fp32
        extra = np.zeros((N, E))
        for r in range(N):
            for j in range(ch.shape[1]):
                if 0 <= ch[r, j] < E:
                    extra[r, ch[r, j]] += abs(gv[r, j])
        tol = tol + U * (ch.shape[1] + 1) * extra
    dtype = {v: k for k, v in TYPES.items()}[x.dtype]
    near(wide(got), want, tol + near_type * np.abs(want) * (1 + near_type) + TINY[dtype], "gradient")
    return got


def upstream(groups, N, k, dtype, seed, vals=True):
    gen = torch.Generator().manual_seed(seed)
    scale = 16.0 * N / groups if dtype == "f16" else 1.0
    gl = torch.randn((groups,), generator=gen) * scale
    gz = torch.randn((groups,), generator=gen) * 0.1 * scale
    gv = torch.randn((N, k), generator=gen) * scale / N if vals else None
    return gl.cuda(), gz.cuda(), gv.cuda() if vals else None


SHAPES = [(1, 1, 1, 1), (1, 2, 1, 1), (3, 3, 2, 1), (64, 4, 2, 1), (33, 8, 2, 1), (35, 8, 8, 5), (1000, 16, 1, 1), (999, 31, 4, 3), (300, 32, 2, 300), (513, 60, 4, 1), (700, 64, 8, 7),
          (260, 65, 6, 2), (129, 100, 5, 1), (500, 128, 8, 4), (90, 160, 6, 1), (101, 255, 12, 1), (222, 256, 8, 2), (64, 257, 3, 1), (77, 500, 10, 7), (50, 512, 8, 1), (30, 513, 9, 1),
          (20, 1000, 40, 4), (9, 1024, 64, 1), (40000, 8, 2, 2), (20001, 24, 3, 3)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,E,k,groups", SHAPES)
@pytest.mark.parametrize("pad,shift,ignored", [(0, 0, 0), (3, 1, 3)])
def test_loss_and_gradient(dtype, N, E, k, groups, pad, shift, ignored):
    R = _gpu()
    for width in (4, 1) if E < 255 else (4,):
        x, cols = inputs(N, E, k, dtype, N + E, pad, shift, ignored, width)
        _, _, _, counts, rows = check_forward(R, x, cols, groups)
        gl, gz, gv = upstream(groups, N, k, dtype, 7 * E)
        check_gradient(R, x, cols, counts, rows, gl)
        check_gradient(R, x, cols, counts, rows, gl, gz, gv)


def test_long_groups():
    R = _gpu()
    for N, E, groups in ((300000, 8, 1), (70001, 64, 1), (65536, 60, 2)):
        x, cols = inputs(N, E, 2, "bf16", N, ignored=8)
        check_forward(R, x, cols, groups)


def test_a_loss_by_one_workgroup():
    """Without scratch memory a group is one workgroup's work."""
    R = _gpu()
    lib = R.load_library()
    x, cols = inputs(30000, 16, 2, "f32", 4)
    got = [torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty((1, 16), device="cuda"), torch.empty((1, 16), dtype=torch.int32, device="cuda"),
           torch.empty(1, dtype=torch.int32, device="cuda")]
    assert R.rtopk_balance_workspace_bytes(30000, 16, torch.float32, 2) > 0
    assert lib.rtopk_balance_loss(x.data_ptr(), 0, 30000, 16, 16, cols.data_ptr(), 4, 2, 1, *[t.data_ptr() for t in got], None, 0, torch.cuda.current_stream().cuda_stream) == 0
    check_forward(R, x, cols, got=got)
    # optional outputs
    again = torch.empty(1, device="cuda")
    assert lib.rtopk_balance_loss(x.data_ptr(), 0, 30000, 16, 16, cols.data_ptr(), 4, 2, 1, again.data_ptr(), None, None, got[3].data_ptr(), got[4].data_ptr(), None, 0,
                                  torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(again, got[0])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_masked_experts_empty_rows_and_values_that_are_no_numbers(dtype):
    R = _gpu()
    N, E, k, groups = 40, 24, 3, 4
    x, cols = inputs(N, E, k, dtype, 5)
    x[:, 20:] = -float("inf")      # experts that are switched off
    cols = torch.topk(x.float(), k, dim=1)[1].to(torch.int32)  # in the order of the values
    x[3] = -float("inf")
    x[4] = torch.finfo(x.dtype).min
    x[5, 0] = torch.finfo(x.dtype).max
    x[12, 3] = float("nan")        # spoils group 1
    x[27, 3] = float("inf")        # and 2
    got = R.rtopk_balance_loss(x, cols, groups)
    assert torch.isnan(got[0][1:3]).all() and torch.isnan(got[1][1:3]).all() and torch.isfinite(got[0][[0, 3]]).all()
    check_forward(R, x[:10], cols[:10])
    check_forward(R, x[30:], cols[30:])
    alone = R.rtopk_balance_loss(x[30:], cols[30:])
    assert torch.equal(alone[2][0], got[2][3])
    gl, gz, gv = upstream(groups, N, k, dtype, 3)
    grad = check_gradient(R, x, cols, got[3], got[4], gl, gz, gv)
    bad = ~torch.isfinite(grad).all(dim=1)
    assert bad.nonzero().flatten().tolist() == [12, 27]


def test_tokens_left_out_and_groups_of_padding():
    R = _gpu()
    N, E, k = 60, 16, 2
    x, cols = inputs(N, E, k, "f32", 6)
    cols[:20] = -1
    cols[20:30, 0] = E  # one of two
    x[7] = float("nan")  # padding may hold anything
    got = check_forward(R, x, cols, 3)
    assert got[0][0] == 0 and got[1][0] == 0 and (got[2][0] == 0).all() and got[4].tolist() == [0, 20, 20]
    gl, gz, gv = upstream(3, N, k, "f32", 3)
    grad = check_gradient(R, x, cols, got[3], got[4], gl, gz, gv)
    assert (grad[:20] == 0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_tokens_left_out_of_a_loss_that_overflowed(dtype):
    """Padding has a gradient of 0 also where a loss scale has made the group's gradients infinite."""
    R = _gpu()
    x, cols = inputs(400, 24, 3, dtype, 1, ignored=4)
    _, _, _, counts, rows = R.rtopk_balance_loss(x, cols, 4)
    out = (cols < 0).all(1)
    bad = torch.tensor([float("inf"), float("nan"), -float("inf"), 1.0], device="cuda")
    for gz, vals in ((None, None), (bad.flip(0).contiguous(), torch.ones((400, 3), device="cuda"))):
        grad = R.rtopk_balance_loss_backward(bad, x, cols, counts, rows, gz, vals)
        assert out.sum() == 100 and (grad[out] == 0).all() and not grad[:100][~out[:100]].isfinite().any()


def test_offsets_beyond_32_bits():
    """The last of two groups of 2^32 logits each behind the other."""
    R = _gpu()
    N, E, k = 1 << 25, 256, 2
    x = torch.zeros((N, E), dtype=torch.bfloat16, device="cuda")
    cols = torch.zeros((N, k), dtype=torch.int32, device="cuda")
    cols[:, 1] = 1
    tail, picked = inputs(N // 2 // 64, E, k, "bf16", 3)
    for i in range(64):
        x[N // 2 + i * tail.shape[0]:][:tail.shape[0]] = tail
        cols[N // 2 + i * tail.shape[0]:][:tail.shape[0]] = picked
    whole = R.rtopk_balance_loss(x, cols, 2)
    assert whole[3][0].tolist() == [N // 2, N // 2] + [0] * (E - 2) and whole[4].tolist() == [N // 2] * 2
    assert torch.equal(whole[3][1], 64 * R.rtopk_balance_loss(tail, picked)[3][0])
    near(wide(whole[0][:1]), [1.0], 200 * U, "loss")  # (equal probabilities, 1 / E each: f_e P_e E sums to 1)
    few = R.rtopk_balance_loss(tail, picked)
    near(wide(whole[0][1:]), wide(few[0]), 240 * U * wide(few[0]), "loss")  # (each within (2 D + 80) U of the definition, as above, D < 20)
    grad = torch.ones((2,), device="cuda") * N
    got = R.rtopk_balance_loss_backward(grad, x, cols, whole[3], whole[4], None, None, x)
    last = R.rtopk_balance_loss_backward(grad[1:], tail, picked, whole[3][1:], whole[4][1:])
    assert torch.equal(got[-tail.shape[0]:], last) and not got[N // 2:].isnan().any()
    assert torch.equal(got[0], got[N // 2 - 1])


def test_no_tokens():
    R = _gpu()
    x, cols = torch.empty((0, 8), device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda")
    loss, z, probs, counts, rows = R.rtopk_balance_loss(x, cols, 3)
    for t in (loss, z, probs, counts, rows):
        assert (t == 0).all()
    assert R.rtopk_balance_loss_backward(loss, x, cols, counts, rows).shape == (0, 8)


def test_the_same_column_twice():
    R = _gpu()
    x, _ = inputs(50, 12, 3, "f32", 6)
    cols = torch.randint(0, 12, (50, 6), generator=torch.Generator().manual_seed(1)).int().cuda()
    cols[0] = 5
    got = check_forward(R, x, cols)
    gl, gz, gv = upstream(1, 50, 6, "f32", 3)
    grad = check_gradient(R, x, cols, got[3], got[4], gl, gz, gv)
    for _ in range(3):
        assert torch.equal(grad, R.rtopk_balance_loss_backward(gl, x, cols, got[3], got[4], gz, gv))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E", [8, 60, 300])
def test_in_the_logits_place(dtype, E):
    R = _gpu()
    x, cols = inputs(333, E, 3, dtype, 6, pad=5, shift=1)
    _, _, _, counts, rows = R.rtopk_balance_loss(x, cols)
    gl, gz, gv = upstream(1, 333, 3, dtype, 3)
    before = x.clone()
    want = R.rtopk_balance_loss_backward(gl, x, cols, counts, rows, gz, gv)
    got = check_gradient(R, x, cols, counts, rows, gl, gz, gv, before=before, grad_logits=x)
    assert got is x and torch.equal(got, want)
    whole = torch.as_strided(x, (333, E + 5), (E + 5, 1))
    assert torch.isnan(whole[:-1, E:]).all()  # what lies between rows is left as it was


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E,bytes", [(7, 4), (33, 1), (96, 4), (256, 1), (523, 4)])
def test_given_outputs_and_what_lies_between_rows(dtype, E, bytes):
    R = _gpu()
    N, k, groups = 90, min(E, 5), 3
    x, cols = inputs(N, E, k, dtype, E, 5, 1, 4, bytes) if bytes == 4 else inputs(N, E, k, dtype, E, 5, 1, 0, bytes)
    if E == 256:
        cols[:, k - 1] = 255
    out = [torch.full(s, 7, dtype=t, device="cuda") for s, t in (((groups,), torch.float32),) * 2 + (((groups, E), torch.float32), ((groups, E), torch.int32), ((groups,), torch.int32))]
    got = R.rtopk_balance_loss(x, cols, groups, *out)
    assert all(a.data_ptr() == b.data_ptr() for a, b in zip(got, out))
    check_forward(R, x, cols, groups, got)
    gl, gz, gv = upstream(groups, N, k, dtype, 3)
    buf = torch.full((N * (E + 3) + 9,), 5.0, dtype=TYPES[dtype], device="cuda")
    to = buf[1:1 + N * (E + 3)].view(N, E + 3)
    for more in ((), (gz, gv)):
        buf.fill_(5.0)
        grad = check_gradient(R, x, cols, got[3], got[4], gl, *more, grad_logits=to[:, :E])
        assert grad.data_ptr() == to.data_ptr() and (to[:, E:] == 5).all() and buf[0] == 5 and (buf[1 + N * (E + 3):] == 5).all()


def test_against_differences():
    R = _gpu()
    x, cols = inputs(24, 10, 2, "f32", 6, scale=1.0)
    base = R.rtopk_balance_loss(x, cols, 2)
    gl, gz, _ = upstream(2, 24, 2, "f32", 9)
    grad = wide(R.rtopk_balance_loss_backward(gl, x, cols, base[3], base[4], gz))
    xh, ch, h = wide(x), cols.cpu().numpy(), 1e-5
    for n, e in ((0, 0), (3, 7), (11, 9), (12, 4), (23, 1)):
        both = []
        for s in (h, -h):
            y = xh.copy()
            y[n, e] += s
            loss, z, _, _, _ = definition.loss(y, ch, 2)
            both.append((loss * wide(gl)).sum() + (z * wide(gz)).sum())
        # differences of 64-bit sums: h^2 of the third derivative, and 1e-16 / h
        assert abs((both[0] - both[1]) / (2 * h) - grad[n, e]) < 1e-8 + 1e-5 * abs(grad[n, e])


def test_a_router_as_it_is_used():
    """Selection, loss and gradient together: picks of the framework's own selection, the gradient of the picked values on the way."""
    R = _gpu()
    N, E, k = 4096, 64, 8
    x, _ = inputs(N, E, k, "f32", 6)
    x = x.contiguous()
    vals, cols = R.rtopk_rowwise_exact(x, k)
    byte_vals, byte_cols = R.rtopk_rowwise_exact_u8(x, k)
    got = check_forward(R, x, cols, 4)
    bytes_ = R.rtopk_balance_loss(x, byte_cols, 4)
    assert all(torch.equal(a, b) for a, b in zip(got, bytes_))
    gl, _, gv = upstream(4, N, k, "f32", 3)
    with_vals = check_gradient(R, x, cols, got[3], got[4], gl, None, gv)
    without = R.rtopk_balance_loss_backward(gl, x, cols, got[3], got[4])
    apart = without + R.rtopk_maxk_backward(gv, cols, E)
    # apart: the product e t of the loss's gradient is rounded (U of it), then its sum with the picked value's (U of that); fused: that sum alone (U again).
    # The two terms may cancel, so the first is no part of the sum's size.
    near(wide(with_vals), wide(apart), U * np.abs(wide(without)) + 2 * U * np.abs(wide(apart)) + 1e-30, "fused")


def test_captured_and_on_other_streams():
    R = _gpu()
    N, E, k = 5000, 32, 4
    x, cols = inputs(N, E, k, "bf16", 6)
    gl, gz, gv = upstream(2, N, k, "bf16", 3)

    def step():
        out = R.rtopk_balance_loss(x, cols, 2)
        return out + (R.rtopk_balance_loss_backward(gl, x, cols, out[3], out[4], gz, gv),)

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out, torch.cuda.Stream()))
    for turn in range(4):
        y, c = inputs(N, E, k, "bf16", 60 + turn)
        x.copy_(y)
        cols.copy_(c)
        torch.cuda.synchronize()
        for g, _, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = step()
        check_forward(R, x, cols, 2, want[:5])
        for _, out, _ in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    R = _gpu()
    x, cols = inputs(12, 8, 2, "f32", 1)
    loss, z, probs, counts, rows = R.rtopk_balance_loss(x, cols)
    for args in ((x.cpu(), cols), (x.double(), cols), (x.t(), cols), (x, cols.long()), (x, cols[:5]), (x, cols.cpu()), (x, cols[:, 0]), (x[0], cols)):
        with pytest.raises(ValueError):
            R.rtopk_balance_loss(*args)
    for groups in (0, -1, 5):
        with pytest.raises(R.RTopKError):
            R.rtopk_balance_loss(x, cols, groups)
    with pytest.raises(R.RTopKError):
        R.rtopk_balance_loss(torch.zeros((2, 1025), device="cuda"), cols[:2])
    with pytest.raises(R.RTopKError):
        R.rtopk_balance_loss(torch.zeros((2, 300), device="cuda"), cols[:2].to(torch.uint8))
    with pytest.raises(R.RTopKError):  # more picks than experts
        R.rtopk_balance_loss(x[:, :1], cols)
    gl = torch.ones(1, device="cuda")
    ok = dict(grad_loss=gl, logits=x, cols=cols, counts=counts, rows=rows)
    R.rtopk_balance_loss_backward(**ok)
    for kw in (dict(grad_loss=torch.ones(2, device="cuda")), dict(counts=counts.long()), dict(counts=counts[0]), dict(counts=counts[:, :4]), dict(rows=rows.float()), dict(grad_z=gl.double()),
               dict(grad_vals=torch.ones((12, 3), device="cuda")), dict(grad_logits=x.half()), dict(grad_logits=torch.empty((12, 9), device="cuda")), dict(cols=cols.long())):
        with pytest.raises(ValueError):
            R.rtopk_balance_loss_backward(**{**ok, **kw})
    with pytest.raises(R.RTopKError):  # over its logits, but not in their place
        R.rtopk_balance_loss_backward(gl, x[:11], cols[:11], counts, rows, grad_logits=x[1:])
