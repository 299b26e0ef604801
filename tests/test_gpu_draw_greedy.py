"""Greedy verification where draft logits are given, which are then not looked at, and calls with scratch memory against calls without.  Tolerances: none, tokens are whole
numbers (tests/test_gpu_draw.py)."""
import pytest

from test_gpu_draw import TYPES, _gpu, block, check_verify, drawn_from, numbers
from test_gpu_draw_many import by_workgroups, near_draft, same

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype,B,G,M", [("f32", 16, 4, 50001), ("f32", 8, 4, 32000), ("f16", 38, 3, 70000), ("bf16", 32, 4, 65536), ("f32", 128, 3, 32000), ("bf16", 3, 2, 500)])
def test_draft_logits_at_temperature_0(dtype, B, G, M):
    R = _gpu()
    target = block((B, G + 1, M), dtype, B)
    draft = near_draft(target, G, 3, 0.3)
    drafts = target[:, :G].float().argmax(-1)
    drafts[::3, G - 1] = 1
    drafts[1::4, 0] = M
    u = numbers((B, G + 1), 2)
    want = check_verify(R, target, drafts, u, None, 0.0)
    draft[::2] = float("nan")
    for T in (0, 0.0):
        same(R.rtopk_verify_drafts(target, drafts, u, draft, T), want)
        same(R.rtopk_verify_drafts(target, drafts, None, draft, T), want)
    same(by_workgroups(R, target, drafts, u, draft, 0.0), want)
    same(R.rtopk_verify_drafts(target, drafts, u, draft, torch.zeros(B, device="cuda")), want)


@pytest.mark.parametrize("dtype,B,G,M", [("bf16", 300, 3, 2500), ("f32", 300, 4, 9000), ("f16", 5, 1, 4097)])
def test_with_and_without_scratch_memory(dtype, B, G, M):
    """The same tokens from one workgroup to a sequence as from many, where there is scratch memory to be without."""
    R = _gpu()
    target = block((B, G + 1, M), dtype, B)
    draft = near_draft(target, G, M)
    drafts = drawn_from(draft, 1.0, B)
    u = numbers((B, G + 1), B)
    for q in (draft, None):
        assert R.rtopk_verify_workspace_bytes(B, G, M, TYPES[dtype], q is not None) > 0
        same(R.rtopk_verify_drafts(target, drafts, u, q), by_workgroups(R, target, drafts, u, q))
