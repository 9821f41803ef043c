"""A student's vocabulary head learns from a teacher's top logits, and its gradient is compressed.

Each step runs the library's calls as a training program would:

    teacher logits            -> gk_vocab_topk      k pairs and the log-sum-exp a row: the teacher's message
    student's h, w, message   -> gk_vocab_distill   loss and the head's gradient, no logits kept
    student's h, w, words     -> gk_vocab_loss      the same for the words themselves
    both gradients            -> gk_sparsify        Gaussian_k with the residual carried over
    pairs                     -> gk_apply_gathered  the step on the head's fp32 weights

    python examples/distill_head.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1911_08772_b200 import binding as gk  # noqa: E402


def train(steps: int = 40, rows: int = 512, width: int = 256, words: int = 4001, k: int = 32, temperature: float = 2.0,
          density: float = 0.01, rate: float = 15.0, seed: int = 0):
    """Returns the mean loss (distillation plus words) of each step.  The body that makes h is left out:
    h is drawn anew each step, the teacher's head is fixed and the student's starts from zero."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    teacher = (torch.randn(words, width, generator=gen, device=dev) * (2.0 / width ** 0.5)).bfloat16()
    master = torch.zeros(words * width, device=dev)              # the student's head in fp32
    residual = torch.zeros_like(master)
    keep = max(1, int(density * master.numel()))
    pairs = (torch.empty(master.numel(), dtype=torch.int32, device=dev), torch.empty(master.numel(), device=dev),
             torch.zeros(1, dtype=torch.int64, device=dev))
    t_idx = torch.empty(rows, k, dtype=torch.int32, device=dev)
    t_val = torch.empty(rows, k, device=dev)
    t_lse, loss, lse = (torch.empty(rows, device=dev) for _ in range(3))
    dw_soft, dw_hard = torch.empty_like(teacher), torch.empty_like(teacher)
    dh = torch.empty(rows, width, dtype=torch.bfloat16, device=dev)     # would go on into the body
    means = []
    for _ in range(steps):
        h = torch.randn(rows, width, generator=gen, device=dev).bfloat16()
        logits = h @ teacher.t()
        gk.gk_vocab_topk(logits, k, t_idx, t_val, lse_out=t_lse, temperature=temperature)
        w = master.view(words, width).bfloat16()
        gk.gk_vocab_distill(h, w, t_idx, t_val, loss, lse, t_lse=t_lse, temperature=temperature, dh=dh, dw=dw_soft)
        mean = loss.mean()
        gk.gk_vocab_loss(h, w, logits.argmax(dim=1), loss, lse, dh=dh, dw=dw_hard)
        means.append(mean + loss.mean())
        grad = (dw_soft.float() + dw_hard.float()).view(-1)
        idx, val, nnz = pairs
        gk.gk_sparsify(grad, residual, keep, idx, val, nnz)
        gk.gk_apply_gathered(master, idx, val, nnz, master.numel(), -rate)
    return torch.stack(means).tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    losses = train(ap.parse_args().steps)
    for i, x in enumerate(losses):
        if i % 5 == 0 or i == len(losses) - 1:
            print(f"step {i:3d}  loss {x:.4f}")


if __name__ == "__main__":
    main()
