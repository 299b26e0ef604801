"""Drawn tokens and verified drafts on the GPU against their definitions in 64 bits (oracle/draw.py, numpy).

Tokens are whole numbers and equal.  A sum's error moves one only where u lies within that error of a border between columns: powers are off by 4 10^-14 of
their value, sums of up to 2^24 of them in trees and runs by less than as much again, so 10^-12 of the row's mass bounds all of it; the inputs
here (fixed seeds) are checked to keep that distance."""
import ctypes

import numpy as np
import pytest

from oracle import draw as definition

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FAR = 1e-12


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_00822_amd as R

    R.load_library()
    return R


def wide(t):
    return t.detach().cpu().double().numpy()


def block(shape, dtype, seed, pad=0, shift=0, scale=3.0):
    """Logits [..., M] on the GPU as a view of a larger buffer of NaN: `pad` columns between rows, `shift` elements before the first."""
    gen = torch.Generator().manual_seed(seed)
    M = shape[-1]
    n = int(np.prod(shape[:-1]))
    buf = torch.full((n * (M + pad) + shift + 64,), float("nan"), dtype=TYPES[dtype])
    x = buf[shift:shift + n * (M + pad)].view(*shape[:-1], M + pad)[..., :M]
    x.copy_((torch.randn(shape, generator=gen) * scale - 2).to(TYPES[dtype]))
    d = buf.cuda()
    return d[shift:shift + n * (M + pad)].view(*shape[:-1], M + pad)[..., :M]


def numbers(shape, seed):
    return torch.rand(shape, generator=torch.Generator().manual_seed(seed)).cuda()


def per_sequence(T, n):
    return [float(v) for v in wide(T)] if isinstance(T, torch.Tensor) else [T] * n


def check_sample(R, x, u, T, **more):
    got = R.rtopk_sample_tokens(x, u, T, **more)
    xh, uh = wide(x), wide(u) if u is not None else np.zeros(x.shape[0])
    for n, t in enumerate(per_sequence(T, x.shape[0])):
        want, near = definition.sample(xh[n], uh[n], t)
        assert near > FAR, ("the input is no test", n, near)
        assert int(got[n]) == want, (n, int(got[n]), want, t, uh[n])
    return got


def check_verify(R, target, drafts, u, draft=None, T=1.0, **more):
    tokens, accepted = R.rtopk_verify_drafts(target, drafts, u, draft, T, **more)
    th, dh, uh, qh = wide(target), drafts.cpu().numpy(), wide(u), wide(draft) if draft is not None else None
    for b, t in enumerate(per_sequence(T, target.shape[0])):
        want, n, near = definition.verify(th[b], dh[b], uh[b], qh[b] if qh is not None else None, t)
        assert near > FAR, ("the input is no test", b, near)
        assert int(accepted[b]) == n and tokens[b].tolist() == want, (b, int(accepted[b]), n, tokens[b].tolist(), want, t)
    assert tokens.dtype == drafts.dtype and accepted.dtype == torch.int32
    return tokens, accepted


def drawn_from(draft, T, seed):
    """Drafts [B, G] drawn from the draft's rows."""
    gen = torch.Generator().manual_seed(seed)
    x = draft.detach().cpu().double()
    noise = -torch.log(-torch.log(torch.rand(x.shape, generator=gen, dtype=torch.float64)))
    T = T.cpu().double().clamp(min=0)[:, None, None] if isinstance(T, torch.Tensor) else T
    return (x + noise * T).argmax(-1).cuda()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,M,pad,shift", [(1, 1, 0, 0), (5, 2, 0, 1), (9, 7, 3, 0), (4, 63, 0, 1), (4, 64, 0, 0), (3, 65, 0, 0), (17, 1000, 1, 0), (6, 1003, 0, 3), (5, 4097, 7, 1),
                                           (3, 8191, 0, 0), (3, 32768, 0, 0), (2, 50001, 0, 1), (2, 131072, 8, 0)])
@pytest.mark.parametrize("T", [1.0, 0.7, 0.0, "mixed"])
def test_sample(dtype, N, M, pad, shift, T):
    R = _gpu()
    x = block((N, M), dtype, 10 * M + N, pad, shift)
    if T == "mixed":
        T = torch.tensor([0.7, 0.0, 1.3, 2.0])[torch.arange(N) % 4].cuda()
    check_sample(R, x, numbers((N,), M + 1), T)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("M", [5, 100, 5000, 40000])
def test_rows_without_a_distribution_and_masks(dtype, M):
    R = _gpu()
    x = block((10, M), dtype, M)
    x[0] = -float("inf")
    x[1, M // 2] = float("nan")
    x[2, M - 1] = float("inf")
    x[3] = -float("inf")
    x[3, M - 1] = -5.0
    x[4, : M - M // 4] = -float("inf")
    x[5] = torch.finfo(x.dtype).min
    x[6] = torch.finfo(x.dtype).min
    x[6, 3] = 1.0
    x[7, 1:] = -float("inf")
    x[8] = 0.0
    u = numbers((10,), M)
    for T in (1.0, 0.25, 0.0):
        if T > 0:
            check_sample(R, x, u, T)
        else:
            want = [definition.sample(row, 0.0, 0.0)[0] for row in wide(x)]
            assert want[2] == M - 1 and want[0] == -1 and want[1] == -1
            assert R.rtopk_sample_tokens(x, None, 0).tolist() == want
    # a row beside them is as if alone
    assert int(R.rtopk_sample_tokens(x, u)[9]) == int(R.rtopk_sample_tokens(x[9:], u[9:])[0])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_numbers_at_the_borders(dtype):
    R = _gpu()
    M = 4096
    x = torch.zeros((8, M), dtype=TYPES[dtype], device="cuda")
    x[:, ::2] = -float("inf")  # 2048 equal ones: every border is a multiple of 2^-11
    last = 1 - 2.0**-24
    u = torch.tensor([0.0, 2.0**-11, 0.5, last, 1.0, 7.0, -3.0, float("nan")], device="cuda")
    assert R.rtopk_sample_tokens(x, u).tolist() == [1, 3, M // 2 + 1, M - 1, M - 1, M - 1, 1, 1]
    # and with a last column that has nothing
    x[:, -3:] = -float("inf")
    x[:, 0] = 0.0
    x[:, 2] = 0.0
    assert R.rtopk_sample_tokens(x, u).tolist()[3:6] == [M - 5] * 3 and R.rtopk_sample_tokens(x, u).tolist()[0] == 0


@pytest.mark.parametrize("T", [float("nan"), -1.0, float("inf"), -float("inf")])
def test_sequences_whose_temperature_is_none(T):
    R = _gpu()
    x = block((3, 2, 500), "f32", 3)
    temps = torch.tensor([1.0, T, 0.0], device="cuda")
    assert R.rtopk_sample_tokens(x[:, 0], numbers((3,), 1), temps).tolist()[1] == -1
    drafts = torch.full((3, 1), 7, device="cuda")
    tokens, accepted = R.rtopk_verify_drafts(x, drafts, numbers((3, 2), 1), x[:, :1], temps)
    assert tokens[1].tolist() == [-1, -1] and int(accepted[1]) == 0
    check = tokens[0].tolist()
    assert check[0] == 7  # the target's own draft is accepted


@pytest.mark.parametrize("T", [1e-6, 1e-30, 1e30])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_far_temperatures(dtype, T):
    R = _gpu()
    x = block((6, 3000), dtype, 8, scale=30.0)
    check_sample(R, x, numbers((6,), 5), T)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("B,M", [(3, 1003), (2, 40000), (300, 16400)])
@pytest.mark.parametrize("T", [3e35, 1e38, 1e300])
def test_masks_at_temperatures_that_make_all_alike(dtype, B, M, T):
    """A masked column has no probability at any temperature, nor does it at one where the type's lowest value would have some."""
    R = _gpu()
    target = block((B, 3, M), dtype, 5)
    draft = block((B, 2, M), dtype, 6)
    target[:, :, ::2] = -float("inf")
    draft[:, :, 1::2] = -float("inf")
    draft[::2, :, : M // 3] = 1.0
    drafts = drawn_from(draft.clamp(min=-1e4), 1.0, 4)
    u = numbers((B, 3), 8)
    some = slice(0, 12)
    check_sample(R, target[some, 0], u[some, 0].contiguous(), T)
    check_verify(R, target[some], drafts[some], u[some], draft[some], T)
    tokens, accepted = R.rtopk_verify_drafts(target, drafts, u, draft, T)
    drawn = tokens.gather(1, accepted.long()[:, None])
    assert (tokens[tokens >= 0] % 2 == 1).all() and (drawn >= 0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("B,G,M,pad,shift", [(1, 1, 2, 0, 0), (3, 2, 5, 1, 1), (7, 1, 64, 0, 0), (5, 4, 1000, 0, 0), (9, 8, 1003, 5, 1), (2, 3, 32000, 0, 0), (2, 5, 50001, 1, 1),
                                             (40, 3, 999, 0, 0), (1, 128, 70, 0, 0)])
@pytest.mark.parametrize("T", [1.0, 0.6, "mixed"])
@pytest.mark.parametrize("noise", [0.3, 2.0])
def test_verify_with_draft_logits(dtype, B, G, M, pad, shift, T, noise):
    R = _gpu()
    target = block((B, G + 1, M), dtype, 100 * G + B, pad, shift)
    draft = block((B, G, M), dtype, 7 * G + B, pad + 1, shift)
    draft.mul_(noise / 3).add_(target[:, :G])
    if T == "mixed":
        T = torch.tensor([0.7, 1.0, 0.0, 1.7])[torch.arange(B) % 4].cuda()
    check_verify(R, target, drawn_from(draft, T, B), numbers((B, G + 1), M), draft, T)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("B,G,M", [(1, 1, 3), (6, 4, 1001), (3, 2, 50001), (70, 3, 500)])
@pytest.mark.parametrize("T", [1.0, 0.0, "mixed"])
def test_verify_of_drafts_that_were_looked_up(dtype, B, G, M, T):
    R = _gpu()
    target = block((B, G + 1, M), dtype, 5 * B)
    if T == "mixed":
        T = torch.tensor([0.7, 0.0, 1.7])[torch.arange(B) % 3].cuda()
    drafts = target[:, :G].float().argmax(-1)  # likely ones, some not
    drafts[::2, -1] = 0
    target.scatter_(2, torch.cat([drafts, drafts[:, :1]], 1)[..., None], 9.0)
    check_verify(R, target, drafts.int() if B == 6 else drafts, numbers((B, G + 1), B), None, T)


def test_fewer_drafts_than_there_is_room_for():
    R = _gpu()
    B, G, M = 8, 5, 3001
    target = block((B, G + 1, M), "bf16", 1)
    draft = target[:, :G].clone()
    drafts = drawn_from(draft, 1.0, 4)
    for b, n in enumerate([0, 1, 2, 3, 4, 5, 0, 5]):
        drafts[b, n:] = [-1, M, -100, 2**40][b % 4]
    target[0, 1:] = float("nan")  # behind the last row that a token is drawn from: not looked at
    draft[0] = float("nan")
    tokens, accepted = check_verify(R, target, drafts, numbers((B, G + 1), 2), draft)
    assert accepted.tolist() == [0, 1, 2, 3, 4, 5, 0, 5]  # the target's own
    assert (tokens[torch.arange(G + 1, device="cuda") > accepted[:, None]] == -1).all()


def test_rows_behind_a_rejected_draft_do_not_count():
    R = _gpu()
    target = block((4, 4, 1000), "f32", 1)
    draft = block((4, 3, 1000), "f32", 2)
    drafts = torch.randint(0, 1000, (4, 3), generator=torch.Generator().manual_seed(1)).cuda()
    u = numbers((4, 4), 3)
    u[:, 0] = 1.0 - 2.0**-24
    draft.scatter_(2, drafts[..., None], 12.0)  # drafts that the target finds unlikely
    want = check_verify(R, target, drafts, u, draft)
    assert want[1].tolist() == [0, 0, 0, 0]
    target[:, 1:] = float("nan")
    draft[:, 1:] = float("nan")
    got = check_verify(R, target, drafts, u, draft)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_the_target_and_the_draft_that_are_no_distributions(dtype):
    R = _gpu()
    B, G, M = 7, 2, 700
    target, draft = block((B, G + 1, M), dtype, 1), block((B, G, M), dtype, 2)
    drafts = torch.full((B, G), 5, device="cuda")
    target[0, 0] = -float("inf")           # no token
    target[1, 0, 9] = float("nan")
    draft[2, 0, 9] = float("nan")
    draft[3, 0] = -float("inf")            # q = 0: accepted where the target has any
    draft[4, 0] = target[4, 0]             # p = q, and a draft that neither has
    target[4, 0, 5] = draft[4, 0, 5] = -float("inf")
    target[5, 0] = -float("inf")           # all of p is on a column
    target[5, 0, 11] = 0.0
    target[6, 1] = float("inf")
    u = numbers((B, G + 1), 4)
    tokens, accepted = check_verify(R, target, drafts, u, draft)
    assert tokens[0, 0] == -1 and tokens[1, 0] == -1 and tokens[2, 0] == -1 and int(accepted[3]) >= 1
    assert int(accepted[4]) == 0 and tokens[4, 0] != 5 and tokens[4, 0] >= 0 and tokens[5, 0] == 11


def test_the_same_numbers_in_any_layout():
    R = _gpu()
    B, G, M = 6, 3, 2501
    target, draft = block((B, G + 1, M), "f16", 1), block((B, G, M), "f16", 2)
    drafts, u = drawn_from(draft, 1.0, 1), numbers((B, G + 1), 5)
    want = check_verify(R, target, drafts, u, draft)
    by_position = target.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    draft_by_position = draft.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    assert not by_position.is_contiguous()
    out, n = torch.empty_like(want[0]), torch.empty_like(want[1])
    got = R.rtopk_verify_drafts(by_position, drafts, u, draft_by_position, out_tokens=out, out_accepted=n)
    assert got[0] is out and got[1] is n and torch.equal(out, want[0]) and torch.equal(n, want[1])
    got = R.rtopk_verify_drafts(target, drafts.int(), u, draft, temperature=torch.ones(B, device="cuda"))
    assert got[0].dtype == torch.int32 and torch.equal(got[0].long(), want[0])
    out32 = torch.empty(B, dtype=torch.int32, device="cuda")
    assert R.rtopk_sample_tokens(target[:, 0], u[:, 0].contiguous(), 1.0, out32) is out32
    assert torch.equal(out32.long(), R.rtopk_sample_tokens(target[:, 0].contiguous(), u[:, 0].contiguous()))


def test_no_sequences_and_no_drafts():
    R = _gpu()
    x = block((3, 1, 100), "f32", 1)
    u = numbers((3, 1), 1)
    tokens, accepted = R.rtopk_verify_drafts(x, torch.empty((3, 0), dtype=torch.int64, device="cuda"), u)
    assert torch.equal(tokens[:, 0], R.rtopk_sample_tokens(x[:, 0], u[:, 0].contiguous())) and accepted.tolist() == [0, 0, 0]
    assert R.rtopk_sample_tokens(x[:0, 0], u[:0, 0].contiguous()).shape == (0,)
    tokens, accepted = R.rtopk_verify_drafts(x[:0], torch.empty((0, 0), dtype=torch.int64, device="cuda"), u[:0])
    assert tokens.shape == (0, 1) and accepted.shape == (0,)


@pytest.mark.parametrize("B,G,M", [(1, 4, 32000), (3, 2, 131072), (300, 2, 1000)])
def test_with_and_without_scratch_memory(B, G, M):
    """The same tokens from one workgroup to a sequence as from many."""
    R = _gpu()
    lib = R.load_library()
    target = block((B, G + 1, M), "bf16", 1)
    draft = (target[:, :G].float() + 0.5 * block((B, G, M), "f32", 2)).bfloat16()
    drafts, u = drawn_from(draft, 1.0, 1), numbers((B, G + 1), 5)
    for q in (draft, None):
        want = R.rtopk_verify_drafts(target, drafts, u, q)
        out, n = torch.empty_like(want[0]), torch.empty_like(want[1])
        status = lib.rtopk_verify_drafts(target.data_ptr(), q.data_ptr() if q is not None else None, 2, B, G, M, (G + 1) * M, M, G * M, M, drafts.data_ptr(), 8, u.data_ptr(), None,
                                         1.0, out.data_ptr(), n.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
        assert status == 0 and torch.equal(out, want[0]) and torch.equal(n, want[1])
    want = R.rtopk_sample_tokens(target[:, 0], u[:, 0].contiguous())
    out, first = torch.empty_like(want), u[:, 0].contiguous()
    assert lib.rtopk_sample_tokens(target.data_ptr(), 2, B, M, (G + 1) * M, first.data_ptr(), None, 1.0, out.data_ptr(), 8, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype,B,G,M", [("bf16", 2, 0, 1 << 24), ("f32", 1, 0, (1 << 24) - 5), ("f16", 1, 1, 3000001), ("bf16", 3, 1, 1200000)])
def test_the_widest_rows(dtype, B, G, M):
    R = _gpu()
    lib = R.load_library()
    target, u = block((B, G + 1, M), dtype, 3), numbers((B, G + 1), 4)
    draft = (target[:, :G].float() + 0.5 * block((B, G, M), "f32", 2)).to(TYPES[dtype]) if G else None
    drafts = draft.argmax(-1) if G else torch.zeros((B, 0), dtype=torch.int64, device="cuda")
    want = check_verify(R, target, drafts, u, draft)
    out, n = torch.empty_like(want[0]), torch.empty_like(want[1])
    status = lib.rtopk_verify_drafts(target.data_ptr(), draft.data_ptr() if G else None, list(TYPES).index(dtype), B, G, M, (G + 1) * M, M, G * M, M, drafts.data_ptr() if G else None, 8, u.data_ptr(),
                                     None, 1.0, out.data_ptr(), n.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
    assert status == 0 and torch.equal(out, want[0]) and torch.equal(n, want[1])


@pytest.mark.parametrize("N,M", [(5, 700), (3, 40000), (600, 9000)])
def test_tokens_of_32_bits_and_what_lies_around_them(N, M):
    R = _gpu()
    x, u = block((N, M), "bf16", 5, pad=3, shift=1), numbers((N,), 6)
    buf = torch.full((N + 2,), 77, dtype=torch.int32, device="cuda")
    got = R.rtopk_sample_tokens(x, u, 0.9, out_tokens=buf[1:N + 1])
    assert got.data_ptr() == buf[1:].data_ptr() and buf[0] == 77 and buf[N + 1] == 77
    assert torch.equal(got.long(), R.rtopk_sample_tokens(x, u, 0.9))
    some = slice(0, 5)
    check_sample(R, x[some], u[some], 0.9)


def test_captured_and_on_other_streams():
    R = _gpu()
    B, G, M = 4, 3, 32000
    target, draft = block((B, G + 1, M), "f32", 1), block((B, G, M), "f32", 2)
    draft.mul_(0.2).add_(target[:, :G])
    drafts, u = drawn_from(draft, 1.0, 1), numbers((B, G + 1), 5)
    first = u[:, 0].contiguous()
    R.rtopk_verify_drafts(target, drafts, u, draft)
    R.rtopk_sample_tokens(target[:, 0], first)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):  # two graphs, run on two streams at once
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = R.rtopk_verify_drafts(target, drafts, u, draft) + (R.rtopk_sample_tokens(target[:, 0], first),)
        graphs.append((g, out, torch.cuda.Stream()))
    for step in range(4):
        target.copy_(block(tuple(target.shape), "f32", 10 + step))
        draft.copy_(target[:, :G] + 0.1 * step)
        u.copy_(numbers((B, G + 1), 20 + step))
        first.copy_(u[:, 0])
        torch.cuda.synchronize()
        for g, _, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = check_verify(R, target, drafts, u, draft) + (check_sample(R, target[:, 0], first, 1.0),)
        for _, out, _ in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    R = _gpu()
    x, d, u = block((2, 3, 50), "f32", 1), torch.zeros((2, 2), dtype=torch.int64, device="cuda"), numbers((2, 3), 1)
    ok = dict(target_logits=x, drafts=d, uniforms=u)
    R.rtopk_verify_drafts(**ok)
    for kw in (dict(target_logits=x[0]), dict(target_logits=x.cpu()), dict(target_logits=x.double()), dict(target_logits=x.transpose(1, 2)), dict(drafts=d[:, :1]), dict(drafts=d.float()),
               dict(drafts=d.cpu()), dict(uniforms=u[:, :2]), dict(uniforms=u.double()), dict(uniforms=None), dict(draft_logits=x), dict(draft_logits=x[:, :2].half()),
               dict(temperature=torch.ones(3, device="cuda")), dict(temperature=torch.ones(2, device="cuda", dtype=torch.float64)), dict(out_tokens=d),
               dict(out_tokens=torch.zeros((2, 3), dtype=torch.int32, device="cuda")), dict(out_accepted=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(target_logits=x[:, :0]),
               dict(target_logits=x[:1].expand(2, 3, 50))):
        with pytest.raises(ValueError):
            R.rtopk_verify_drafts(**{**ok, **kw})
    for T in (-1.0, float("nan"), float("inf")):
        with pytest.raises(R.RTopKError):
            R.rtopk_verify_drafts(**ok, temperature=T)
        with pytest.raises(R.RTopKError):
            R.rtopk_sample_tokens(x[0], u[0], T)
    for args in ((x, u[0]), (x[0], u[0, :2]), (x[0], u[0].half()), (x[0].t(), u[0]), (x[0], None)):
        with pytest.raises(ValueError):
            R.rtopk_sample_tokens(*args)
    with pytest.raises(R.RTopKError):  # 129 drafts
        R.rtopk_verify_drafts(torch.zeros((1, 130, 4), device="cuda"), torch.zeros((1, 129), dtype=torch.int64, device="cuda"), numbers((1, 130), 1))
    with pytest.raises(R.RTopKError):  # outputs over inputs
        R.rtopk_sample_tokens(x[0], u[0], out_tokens=x.view(-1).view(torch.int32)[:3])
    assert ctypes.sizeof(ctypes.c_double) == 8
