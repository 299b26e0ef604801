"""A student language-model head trained on a teacher's top logits, with everything on rows of logits through this library:

  teacher   rtopk_token_logprobs: the top alternatives of each position, as log probabilities and columns (all that is kept of the teacher)
  student   rtopk_distill_with_grad: loss and gradient of the logits in one pass over them, the gradient in the logits' place; the head's own
            gradient is a matrix product with it
  watched   rtopk_token_logprobs: log probability of the teacher's first choice, entropy and agreement of the two first choices

    python examples/distill_student.py --vocabulary 32000 --steps 50
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2409_00822_amd as R  # noqa: E402


def train(vocabulary=32000, hidden=256, positions=1024, k=32, steps=50, rate=5.0, temperature=1.0, dtype=torch.bfloat16, seed=0):
    """Returns a dict of lists, an entry for each step: loss, logprob, entropy, agreement."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    features = torch.randn((positions, hidden), device="cuda", generator=gen).to(dtype)
    teacher_head = (torch.randn((hidden, vocabulary), device="cuda", generator=gen) * (3 / hidden**0.5)).to(dtype)
    student_head = torch.zeros((hidden, vocabulary), device="cuda")

    teacher = features @ teacher_head
    first = torch.zeros((positions,), dtype=torch.int64, device="cuda")
    _, _, _, teacher_logprobs, teacher_cols = R.rtopk_token_logprobs(teacher, first, k, temperature)
    first = teacher_cols[:, 0].contiguous()

    weights = torch.full((positions,), 1 / positions, device="cuda")
    seen = {"loss": [], "logprob": [], "entropy": [], "agreement": []}
    for _ in range(steps):
        logits = features @ student_head.to(dtype)
        logprob, entropy, _, _, best = R.rtopk_token_logprobs(logits, first, 1, temperature)
        loss, grad = R.rtopk_distill_with_grad(weights, logits, teacher_logprobs, teacher_cols, temperature, log_probs=True, grad_logits=logits)
        student_head.sub_(rate * positions / hidden * (features.t() @ grad).float())
        for name, value in (("loss", loss.mean()), ("logprob", logprob.mean()), ("entropy", entropy.mean()), ("agreement", (best[:, 0] == first).float().mean())):
            seen[name].append(value)
    return {name: torch.stack(values).tolist() for name, values in seen.items()}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("vocabulary", 32000), ("hidden", 256), ("positions", 1024), ("k", 32), ("steps", 50)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--temperature", type=float, default=1.0)
    seen = train(**vars(ap.parse_args()))
    steps = len(seen["loss"])
    for i in sorted({*range(0, steps, max(1, steps // 10)), steps - 1}):
        print("step %4d  " % i + "  ".join("%s %8.4f" % (name, values[i]) for name, values in seen.items()))


if __name__ == "__main__":
    main()
