"""Verified drafts of many sequences, whose drafts are tested in fp32 beforehand, rows that end with their allocation, and decoding with drafts as a program does it.
Tolerances: none, tokens are whole numbers (tests/test_gpu_draw.py)."""
import numpy as np
import pytest

from oracle import draw as definition
from test_gpu_draw import TYPES, _gpu, block, check_sample, check_verify, drawn_from, numbers, wide

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def by_workgroups(R, target, drafts, u, draft=None, T=1.0):
    """The same call without scratch memory: one workgroup to a sequence, all in 64 bits."""
    lib = R.load_library()
    B, P, M = target.shape
    dtype = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}[target.dtype]
    out, n = torch.empty((B, P), dtype=drafts.dtype, device="cuda"), torch.empty((B,), dtype=torch.int32, device="cuda")
    per = isinstance(T, torch.Tensor)
    status = lib.rtopk_verify_drafts(target.data_ptr(), draft.data_ptr() if draft is not None else None, dtype, B, P - 1, M, target.stride(0), target.stride(1),
                                     draft.stride(0) if draft is not None else 0, draft.stride(1) if draft is not None else 0, drafts.data_ptr(), drafts.element_size(), u.data_ptr(),
                                     T.data_ptr() if per else None, 1.0 if per else T, out.data_ptr(), n.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
    assert status == 0
    return out, n


def same(got, want):
    assert torch.equal(got[1], want[1]) and torch.equal(got[0], want[0]), (got[1] != want[1]).nonzero()[:4].tolist()


def near_draft(target, G, seed, noise=0.6):
    draft = torch.randn((target.shape[0], G, target.shape[2]), generator=torch.Generator().manual_seed(seed)).cuda()
    return draft.mul_(noise).add_(target[:, :G]).to(target.dtype)


SIZES = [("bf16", 300, 2, 20000), ("f16", 200, 3, 16385), ("f32", 130, 4, 32001), ("bf16", 90, 6, 16384), ("bf16", 1100, 3, 2051), ("bf16", 16400, 3, 2500)]


@pytest.mark.parametrize("dtype,B,G,M", SIZES)
@pytest.mark.parametrize("T", [1.0, "mixed"])
def test_many_sequences(dtype, B, G, M, T):
    R = _gpu()
    target = block((B, G + 1, M), dtype, B)
    draft = near_draft(target, G, M)
    if T == "mixed":
        T = torch.tensor([0.7, 1.0, 0.0, 1.7, 0.9])[torch.arange(B) % 5].cuda()
    drafts = drawn_from(draft, T, B)
    drafts[::7, 1:] = -1  # some have fewer
    drafts[3::50, 0] = M
    u = numbers((B, G + 1), B)
    got = R.rtopk_verify_drafts(target, drafts, u, draft, T)
    same(got, by_workgroups(R, target, drafts, u, draft, T))
    pick = torch.arange(0, B, 11, device="cuda")  # (the definition of some)
    some = R.rtopk_verify_drafts(target, drafts, u, draft, T)
    part = check_verify(R, target[pick].contiguous(), drafts[pick].contiguous(), u[pick].contiguous(), draft[pick].contiguous(), T[pick].contiguous() if isinstance(T, torch.Tensor) else T)
    same((some[0][pick], some[1][pick]), part)
    assert 0 < int(got[1].sum()) < B * G


@pytest.mark.parametrize("dtype,B,G,M", [("bf16", 300, 4, 20001), ("f32", 260, 3, 32000)])
def test_many_sequences_with_looked_up_drafts(dtype, B, G, M):
    R = _gpu()
    target = block((B, G + 1, M), dtype, B)
    drafts = target[:, :G].float().argmax(-1)
    drafts[1::3] = torch.randint(0, M, drafts[1::3].shape, generator=torch.Generator().manual_seed(1)).cuda()
    target.scatter_(2, torch.cat([drafts, drafts[:, :1]], 1)[..., None], 9.0)
    u = numbers((B, G + 1), B)
    for T in (1.0, 0.0, torch.tensor([0.7, 0.0, 1.7])[torch.arange(B) % 3].cuda()):
        got = R.rtopk_verify_drafts(target, drafts, u, None, T)
        same(got, by_workgroups(R, target, drafts, u, None, T))
        rows = slice(0, 20)
        check_verify(R, target[rows], drafts[rows], u[rows], None, T[rows].contiguous() if isinstance(T, torch.Tensor) else T)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_many_sequences_with_masks_and_far_values(dtype):
    """Masked columns, rows that are no distributions, logits and temperatures whose powers leave what is summed about 0."""
    R = _gpu()
    B, G, M = 220, 2, 16500
    target = block((B, G + 1, M), dtype, 5)
    draft = near_draft(target, G, 6)
    target[:, :, M - M // 8:] = -float("inf")
    draft[:, :, M - M // 8:] = -float("inf")
    drafts = drawn_from(draft, 1.0, 4)
    target[5, 0] = -float("inf")
    target[6, 0, 9] = float("nan")
    draft[7, 0, 9] = float("nan")
    draft[8, 0] = -float("inf")
    target[9, 1] = float("inf")
    target[10:20] += 2000 if dtype != "bf16" else 2048
    draft[10:20] += 2000 if dtype != "bf16" else 2048
    target[20:30] -= 1500 if dtype != "bf16" else 2048
    draft[30:34] -= 1500
    target[34] = torch.finfo(target.dtype).min
    draft[35] = torch.finfo(target.dtype).min
    T = torch.ones(B)
    T[40:50] = 1e-3
    T[50:60] = 1e-30
    T[60:64] = 1e30
    T[64:70] = torch.tensor([0.0, float("nan"), -1.0, float("inf"), 1e-40, 0.0])
    T = T.cuda()
    u = numbers((B, G + 1), 8)
    got = R.rtopk_verify_drafts(target, drafts, u, draft, T)
    same(got, by_workgroups(R, target, drafts, u, draft, T))
    th, dh, uh, qh = wide(target[:72]), drafts[:72].cpu().numpy(), wide(u[:72]), wide(draft[:72])
    for b in range(72):
        want, n, near = definition.verify(th[b], dh[b], uh[b], qh[b], float(T[b]))
        if near > 1e-12:
            assert int(got[1][b]) == n and got[0][b].tolist() == want, (b, got[0][b].tolist(), want)


def test_numbers_at_the_tests_border():
    """u as near p / q as fp32 has it: the 32-bit test leaves these to the 64-bit one."""
    R = _gpu()
    B, G, M = 300, 2, 20000
    target = block((B, G + 1, M), "f32", 3)
    draft = near_draft(target, G, 4, 1.0)
    drafts = drawn_from(draft, 1.0, 4)

    def share(x):  # (by elementary operations: a library softmax of 64-bit rows as wide as these has fp32's accuracy on this GPU, 9e-7, against 3e-15 on the CPU)
        e = torch.exp(x.double() - x.double().amax(-1, keepdim=True))
        return (e / e.sum(-1, keepdim=True)).gather(2, drafts[..., None])[..., 0]

    p, q = share(target[:, :G]), share(draft)
    u = numbers((B, G + 1), 8)
    ratio = (p / q).float()
    ratio = torch.where(torch.arange(B, device="cuda")[:, None] % 2 == 0, torch.nextafter(ratio, torch.zeros_like(ratio)), torch.nextafter(ratio, torch.full_like(ratio, 9.0)))
    u[:, :G] = torch.where(ratio < 1, ratio, u[:, :G])
    got = R.rtopk_verify_drafts(target, drafts, u, draft)
    same(got, by_workgroups(R, target, drafts, u, draft))
    accepted = (u[:, 0].double() * q[:, 0] < p[:, 0])
    assert torch.equal(got[1] > 0, accepted) and 0 < int(accepted.sum()) < B


@pytest.mark.parametrize("dtype,M", [("f32", 32768), ("bf16", 40001)])
def test_rows_alike_but_for_two_columns(dtype, M):
    """p and q have the same ratio at all columns but two; what is left of p - q is some 10^-7 of the row at one of them and as much at all others together, or
    at that one alone: fp32 sums know neither."""
    R = _gpu()
    B, G = 600, 1
    g = torch.Generator().manual_seed(7)
    target = block((B, G + 1, M), dtype, 3)
    cols = torch.stack([torch.randperm(M, generator=g)[:2] for _ in range(B)]).cuda()  # the draft, raised in q; another one, lowered in it
    low = (torch.randint(-20, 0, (B, 2), generator=g) / 4.0 - 1).cuda()
    more = (torch.randint(1, 9, (B, 2), generator=g) / 4.0).cuda()
    target[:, 0].scatter_(1, cols, low.to(target.dtype))
    draft = target[:, :1].clone()
    draft[:, 0].scatter_(1, cols, (low + more * torch.tensor([1.0, -1.0], device="cuda")).to(target.dtype))
    drafts = cols[:, :1].contiguous()
    u = numbers((B, G + 1), 8)
    u[:, 0] = 1 - 2.0**-24
    tokens, accepted = R.rtopk_verify_drafts(target, drafts, u, draft)
    same((tokens, accepted), by_workgroups(R, target, drafts, u, draft))
    assert (accepted == 0).all()
    alone = tokens[:, 0] == cols[:, 1]
    assert B // 10 < int(alone.sum()) < B - B // 10


def test_the_target_as_its_own_draft():
    R = _gpu()
    B, G, M = 300, 2, 20000
    target = block((B, G + 1, M), "bf16", 3)
    drafts = drawn_from(target[:, :G], 1.0, 4)
    u = numbers((B, G + 1), 8)
    u[:, 0] = 1 - 2.0**-24
    tokens, accepted = R.rtopk_verify_drafts(target, drafts, u, target[:, :G])  # (a view of the target)
    assert (accepted == G).all() and torch.equal(tokens[:, :G], drafts)
    assert torch.equal(tokens[:, G], R.rtopk_sample_tokens(target[:, G], u[:, G].contiguous()))


def test_captured():
    R = _gpu()
    B, G, M = 300, 2, 20000
    target = block((B, G + 1, M), "bf16", 3)
    draft = near_draft(target, G, 4)
    drafts, u = drawn_from(draft, 1.0, 4), numbers((B, G + 1), 8)
    R.rtopk_verify_drafts(target, drafts, u, draft)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = R.rtopk_verify_drafts(target, drafts, u, draft)
    for step in range(4):
        u.copy_(numbers((B, G + 1), 20 + step))
        target.copy_(block((B, G + 1, M), "bf16", 30 + step) if step % 2 else draft[:, [0] * (G + 1)])
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        same(out, R.rtopk_verify_drafts(target, drafts, u, draft))
        same(out, by_workgroups(R, target, drafts, u, draft))


@pytest.mark.parametrize("dtype,N,M", [("bf16", 4096, 32000), ("f16", 2048, 33792 + 512), ("f32", 1024, 17408 + 1024), ("bf16", 16384, 1024), ("f32", 8192, 2304)])
def test_rows_that_end_with_their_allocation(dtype, N, M):
    """A whole number of 2 MiB: what lies behind the last row is nobody's."""
    R = _gpu()
    size = 4 if dtype == "f32" else 2
    assert N * M * size % (1 << 21) == 0
    x = torch.empty((N, M), dtype=TYPES[dtype], device="cuda").normal_().mul_(3)
    u = numbers((N,), 1)
    got = R.rtopk_sample_tokens(x, u)
    check_sample(R, x[-3:], u[-3:].contiguous(), 1.0)
    assert torch.equal(got[-3:], R.rtopk_sample_tokens(x[-3:], u[-3:].contiguous()))


def test_offsets_beyond_32_bits():
    R = _gpu()
    # rows: one behind the other, and far apart
    N, M = 66000, 65536
    x = torch.full((N, M), -float("inf"), dtype=torch.bfloat16, device="cuda")
    x[-5:] = block((5, M), "bf16", 1)
    u = numbers((N,), 1)
    got = R.rtopk_sample_tokens(x, u)
    assert (got[:-5] == -1).all()
    assert torch.equal(got[-5:], check_sample(R, x[-5:], u[-5:].contiguous(), 1.0))
    # sequences
    flat = x.view(-1)
    for B, G, M, seq, pos in ((2, 2, 40000, 1 << 31, 1 << 29), (512, 1, 16500, (1 << 23) + 8, 1 << 22), (2, 1, 700, (1 << 32) - (1 << 29), 1 << 28)):
        assert (B - 1) * seq + G * pos + M <= flat.numel()
        target = torch.as_strided(flat, (B, G + 1, M), (seq, pos, 1))
        target.copy_(block((B, G + 1, M), "bf16", 2))
        draft = torch.as_strided(flat, (B, G, M), (seq, pos, 1), M + 3)
        draft.copy_(near_draft(target, G, 3))
        drafts, u = drawn_from(draft, 1.0, 4), numbers((B, G + 1), 5)
        same(R.rtopk_verify_drafts(target, drafts, u, draft), R.rtopk_verify_drafts(target.contiguous(), drafts, u, draft.contiguous()))


def test_more_sequences_than_a_launch_has():
    R = _gpu()
    B, G, M = 66000, 1, 4100
    torch.manual_seed(5)
    target = torch.empty((B, G + 1, M), dtype=torch.bfloat16, device="cuda").normal_().mul_(3)
    draft = target[:, :G] + torch.empty((B, G, M), dtype=torch.bfloat16, device="cuda").normal_()
    drafts, u = draft.argmax(-1), numbers((B, G + 1), 5)
    got = R.rtopk_verify_drafts(target, drafts, u, draft)
    same(got, by_workgroups(R, target, drafts, u, draft))
    last = slice(B - 600, B)
    check_verify(R, target[last], drafts[last], u[last], draft[last])
    assert torch.equal(got[0][last], R.rtopk_verify_drafts(target[last], drafts[last], u[last], draft[last])[0])


def test_decoding_with_drafts():
    """A target and a draft model (a table of logits by the last token) that decode together.  At temperature 0 the text is the target's own; with random numbers the drafted
    calls are those of the definitions."""
    R = _gpu()
    B, G, M, steps = 6, 3, 3001, 8
    model, small = block((M, M), "bf16", 1), block((M, M), "bf16", 2)
    small.mul_(0.1).add_(model)
    for T in (0.0, 0.8):
        last = torch.arange(B, device="cuda") * 17
        text = [[int(t)] for t in last]
        for step in range(steps):
            u = numbers((B, G + 1), 100 * step + 1)
            more = numbers((G, B), 100 * step + 2)
            drafts, rows, at = [], [], last
            for i in range(G):
                rows.append(small[at])
                at = R.rtopk_sample_tokens(rows[-1], more[i], T)
                drafts.append(at)
            drafts = torch.stack(drafts, 1)
            target = model[torch.cat([last[:, None], drafts], 1)]
            tokens, accepted = check_verify(R, target, drafts, u, torch.stack(rows, 1), T)
            for b in range(B):
                text[b] += tokens[b, : int(accepted[b]) + 1].tolist()
            last = tokens.gather(1, accepted.long()[:, None])[:, 0]
        if T == 0.0:
            at = torch.arange(B, device="cuda") * 17
            for i in range(1, min(len(t) for t in text)):
                at = R.rtopk_sample_tokens(model[at], None, 0)
                assert at.tolist() == [t[i] for t in text]
        assert all(len(t) > steps for t in text)
