"""Scratch memory of drawn tokens and verified drafts, without a GPU: what rtopk_verify_workspace_bytes asks for is enough for the layout of every call that it is
asked for, and is nothing where a sequence is one workgroup's."""
import os

import pytest

F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def size():
    import paper_2409_00822_amd as R

    if not os.path.exists(R.lib_path()):
        from paper_2409_00822_amd import build

        build.build()
    return R.load_library().rtopk_verify_workspace_bytes


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_draft_logits_at_temperature_0(size, dtype):
    """At a temperature of 0 draft logits are not looked at, so that the call's layout is that of drafts that were looked up."""
    short = []
    for G in (1, 2, 3, 4, 5, 6, 7, 8, 31, 128):
        for B in (1, 2, 3, 5, 8, 16, 20, 32, 38, 63, 64, 100, 128, 200, 256, 300, 511, 512, 513, 1024, 4096, 16385):
            for M in (1, 1000, 2049, 4097, 8000, 16383, 16384, 32000, 50001, 100000, 131072, 262144, 1 << 20, (1 << 20) + 1, 1 << 24):
                if size(B, G, M, dtype, 1) < size(B, G, M, dtype, 0):
                    short.append((B, G, M))
    assert not short, (len(short), short[:5])


def test_which_calls_have_some(size):
    for spread in ((1, 0, 131072, BF16, 0), (64, 0, 32000, F32, 0), (1, 4, 32000, F32, 1), (64, 3, 50001, F16, 0), (256, 7, 131072, BF16, 1), (300, 3, 2500, BF16, 0), (300, 3, 2500, BF16, 1)):
        assert size(*spread) > 0, spread
    for one_workgroup in ((1, 0, 8192, BF16, 0), (16385, 0, 131072, F32, 0), (300, 2, 1000, BF16, 1), (300, 2, 1000, BF16, 0), (4096, 4, 1000, F32, 1), (512, 1, (1 << 20) + 1, F32, 1)):
        assert size(*one_workgroup) == 0, one_workgroup
