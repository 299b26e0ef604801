"""The example that runs the operators on rows of logits together: a student learns from a teacher's top logits."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_a_student_learns_from_the_teachers_list():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import distill_student
    finally:
        sys.path.pop(0)
    for dtype in (torch.bfloat16, torch.float32):
        seen = distill_student.train(vocabulary=5003, hidden=64, positions=300, k=16, steps=30, dtype=dtype)
        assert seen["loss"][-1] < 0.5 * seen["loss"][0] and seen["logprob"][-1] > seen["logprob"][0] + 1
        assert seen["agreement"][-1] > 0.8 and seen["entropy"][-1] < seen["entropy"][0]


def test_the_example_runs_as_a_program():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    done = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "distill_student.py"), "--vocabulary", "2000", "--steps", "3", "--positions", "64"],
                          capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and "step    2" in done.stdout, done.stderr[-2000:]
