"""Rows with signalling NaNs (quiet bit clear): the instructions that take maxima return a NaN for them, not the other operand.  Such a row's alternatives are
columns of the row all the same, and other rows are not touched."""
import pytest
from test_gpu_logits import _gpu, check_forward, rows, torch, whole

pytestmark = pytest.mark.gpu

BITS = {"f32": (torch.int32, 0x7FA00001), "f16": (torch.int16, 0x7D01), "bf16": (torch.int16, 0x7FA1)}


def put(x, dtype, where):
    """A signalling NaN at x's places, by its bits."""
    whole_numbers, bits = BITS[dtype]
    x.view(whole_numbers)[where] = bits
    assert torch.isnan(x[where]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,M,k", [(4, 1, 1), (4, 8, 8), (4, 9, 9), (4, 20, 20), (4, 100, 100), (4, 129, 128), (4, 600, 128), (300, 33, 33), (300, 128, 128), (600, 20, 20), (600, 100, 100),
                                   (600, 131, 128), (5000, 32, 32), (4, 5000, 20), (3, 140001, 20)])
def test_alternatives_are_columns_of_the_row(dtype, N, M, k):
    R = _gpu()
    x, xh = rows(N, M, dtype, seed=N + M, pad=3, shift=1)
    kept = x.clone()
    put(x, dtype, (1, slice(M // 2, M // 2 + 1)))  # one, every third, all; the last rows stay as they were
    put(x, dtype, (2, slice(0, None, 3)))
    if N > 3:
        put(x, dtype, (3, slice(None)))
    bad = [1, 2, 3] if N > 3 else [1, 2]
    good = [n for n in (0, *range(4, min(N, 12)), N - 1) if n not in bad]
    t = torch.zeros((N, 1), dtype=torch.int64, device="cuda")
    for got in (R.rtopk_token_logprobs(x, t, k), whole(R, x, t, k)):
        check_forward(R, kept[good], xh[good], t[good], k, got=[g[good] for g in got])
        for n in bad:
            cols = got[4][n].cpu().tolist()
            assert min(cols) >= 0 and max(cols) < M and len(set(cols)) == k, (n, cols)
            assert torch.isnan(got[1][n]) and torch.isnan(got[2][n]) and torch.isnan(got[3][n]).all()
