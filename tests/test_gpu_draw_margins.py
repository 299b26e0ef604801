"""Drafts that fp32 sums decide on, at random numbers as near u q = p as these sums may be off, or nearer: rows on which their roundings add up.  What is accepted is what the
definition in 64 bits accepts, which is off by less than 10^-12 of the values and from all of the numbers here by more than that."""
import numpy as np
import pytest

from test_gpu_draw import TYPES, _gpu
from test_gpu_draw_many import by_workgroups, same

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def mass(row):
    """sum exp(x - max x) of a row in 64 bits, and the maximum."""
    x = row.double()
    return float(torch.exp(x - x.max()).sum()), float(x.max())


def check_around(R, target_row, draft_row, B, units):
    """B sequences with one draft, all of the same rows: u goes from `units` 2^-24 of p / q below it to as much above."""
    M, dtype = target_row.numel(), target_row.dtype
    S_p, m_p = mass(target_row)
    S_q, m_q = mass(draft_row) if draft_row is not None else (1.0, 0.0)
    ratio = torch.exp(target_row.double() - m_p) / S_p
    q = torch.exp(draft_row.double() - m_q) / S_q if draft_row is not None else torch.ones((M,), dtype=torch.float64, device="cuda")
    ratio = torch.where(q > 0, ratio / q, torch.zeros_like(ratio))
    d = int(torch.where(ratio < 0.99, ratio, torch.zeros_like(ratio)).argmax())
    want = float(ratio[d])
    assert 0 < want < 0.99
    u = (want * (1 + torch.linspace(-units, units, B, dtype=torch.float64) * 2.0**-24)).float()
    uq = u.double().numpy()
    assert np.abs(uq / want - 1).min() > 1e-12
    rows = lambda row: torch.as_strided(row.repeat(B + 1), (B, 2, M), (M, M, 1))  # (a sequence's second row is the next one's first)
    target = rows(target_row)
    draft = rows(draft_row)[:, :1] if draft_row is not None else None
    drafts = torch.full((B, 1), d, device="cuda")
    uniforms = torch.stack([u, torch.linspace(0.05, 0.95, B)], 1).cuda().contiguous()
    assert R.rtopk_verify_workspace_bytes(B, 1, M, dtype, draft is not None) > 0
    got = R.rtopk_verify_drafts(target, drafts, uniforms, draft)
    accepted = torch.from_numpy((uq < want).astype(np.int32)).cuda()
    wrong = (got[1] != accepted).nonzero().flatten().tolist()
    assert not wrong, (len(wrong), [round((uq[i] / want - 1) * 2**24) for i in wrong[:3] + wrong[-3:]])
    same(got, by_workgroups(R, target, drafts, uniforms, draft))
    assert B // 4 < int(accepted.sum()) < B - B // 4


def one_sided(steps, sign):
    """Eighths below the maximum, one for each four terms that a thread adds one behind the other: those whose fp32 sum is rounded up (down: sign -1) most."""
    f = np.float32
    k = np.arange(1, 41)
    e = np.exp2((-k.astype(f) / f(8) * f(1.44269504088896340736)).astype(np.float64)).astype(f)
    s, used = f(0), []
    for _ in range(steps):
        t = np.full(k.shape, s, dtype=f)
        for _ in range(4):
            t = t + e
        at = int(np.argmax(sign * (t.astype(np.float64) - s - 4 * e.astype(np.float64)) / e))
        used.append(k[at])
        s = t[at]
    return np.array(used)


@pytest.mark.parametrize("B,waves", [(513, 4), (260, 8), (200, 16)])
@pytest.mark.parametrize("looked_up", [False, True])
def test_maxima_far_from_zero(B, waves, looked_up):
    """Rows about 2^20, whose fp32 sums are taken one term behind the other: 4096 for a thread of four wavefronts."""
    R = _gpu()
    M = 1 << 20
    chunk = np.arange(M // 4) // (64 * waves)  # (a load's four columns go to one thread)

    def row(sign, top):
        x = 2.0**20 - one_sided(M // (256 * waves), sign)[chunk] / 8.0
        x = np.repeat(x, 4)
        x[0] = 2.0**20 - top / 8.0  # the draft
        x[5] = 2.0**20
        return torch.from_numpy(x.astype(np.float32)).cuda()

    check_around(R, row(-1, 4), None if looked_up else row(1, 0), B, 2600)


@pytest.mark.parametrize("dtype,B,M", [("f32", 513, 1 << 20), ("f32", 300, 1 << 20), ("f32", 150, 1 << 20), ("bf16", 520, 1 << 20), ("f16", 600, 300001), ("f32", 1100, 16384)])
@pytest.mark.parametrize("step", [0.0078125, 0.25])
def test_maxima_that_rise_all_along(dtype, B, M, step):
    """Each batch of loads has a new maximum, so that the sums are scaled before each."""
    R = _gpu()
    gen = torch.Generator().manual_seed(M)
    at = torch.arange(M) // 2048
    up = (at * step) % 16.0 - 8.0
    target = (up - 3 * torch.rand((M,), generator=gen)).to(TYPES[dtype]).cuda()
    draft = (up * 0.5 - 2 * torch.rand((M,), generator=gen)).to(TYPES[dtype]).cuda()
    check_around(R, target, draft, B, 2600)
    check_around(R, target, None, B, 1500)
