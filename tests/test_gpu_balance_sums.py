"""Sums over tokens of a router's balance loss: over at most 64 terms in fp32, in 64 bits beyond.

The tokens of one share of lanes have all their probability on expert 0, the others so little that a sum with the former's 64 rounds it away in fp32 in each step, but
not in the end: 0.98 (1 - 1 / shares) of a unit of 64's last place.  Only the output's rounding, U = 2^-24, remains (that of the small ones' own sums is U^2)."""
import math

import numpy as np
import pytest

from oracle import balance as definition
from test_gpu_balance import TYPES, U, _gpu, wide

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E,shares", [(2, 64), (3, 64), (4, 64), (8, 32), (9, 16), (16, 32), (64, 8), (128, 4)])  # (fp32: as the lanes are laid out)
@pytest.mark.parametrize("rounds", [1, 3])
def test_small_terms_beside_large_ones(dtype, E, shares, rounds):
    R = _gpu()
    lib = R.load_library()
    N = 4 * 64 * shares * rounds
    x = torch.full((N, E), -float("inf"))
    x[:, 1] = 0.0
    x[:, 0] = -math.log(2.0**23 * shares / 0.98)
    x[::shares, 0] = 0.0
    x[::shares, 1] = -float("inf")
    x = x.to(TYPES[dtype]).cuda()
    cols = torch.zeros((N, 1), dtype=torch.int32, device="cuda")
    got = [torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty((1, E), device="cuda"), torch.empty((1, E), dtype=torch.int32, device="cuda"),
           torch.empty(1, dtype=torch.int32, device="cuda")]
    assert lib.rtopk_balance_loss(x.data_ptr(), list(TYPES).index(dtype), N, E, E, cols.data_ptr(), 4, 1, 1, *[t.data_ptr() for t in got], None, 0,
                                  torch.cuda.current_stream().cuda_stream) == 0  # (without scratch memory: by one workgroup)
    loss, _, probs, counts, rows = definition.loss(wide(x), cols.cpu().numpy().astype(np.int64), 1)
    assert got[3].tolist() == counts.tolist() and got[4].tolist() == rows.tolist()
    for what, a, b in (("probability", wide(got[2])[0, 0], probs[0, 0]), ("loss", wide(got[0])[0], loss[0])):
        assert abs(a - b) <= U * b * (1 + 2.0**-10), (what, (a - b) / b / U)
    again = R.rtopk_balance_loss(x, cols)  # (by many)
    assert abs(wide(again[2])[0, 0] - probs[0, 0]) <= U * probs[0, 0] * (1 + 2.0**-10)
