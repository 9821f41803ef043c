"""A vocabulary head learns from rewards, its gradients clipped and compressed.

Each step runs the library's calls as a training program would:

    logits of the rollouts     -> gk_vocab_logprob       log probability of each sampled token, entropy, likely others
    advantages, entropy bonus  -> gk_vocab_logprob_grad  the gradient at the logits
    gradients of all tensors   -> gk_grad_norm           what a log shows, tensor by tensor
                               -> gk_grad_clip           clipped into one fp32 vector, 16-bit and fp32 tensors alike
    that vector                -> gk_sparsify            Gaussian_k with the residual carried over
    pairs                      -> gk_apply_gathered      the step on the fp32 weights

    python examples/policy_head.py [--steps N]
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


class Policy:
    """logits = (h scaled by gain) w^T + bias, the weights in fp32 and one vector; w is multiplied in bf16."""

    def __init__(self, words: int, width: int, device):
        self.words, self.width = words, width
        self.weights = torch.zeros(words * width + words + width, device=device)
        self.residual = torch.zeros_like(self.weights)
        self.weights[-width:] = 1.0
        self.dw = torch.empty(words, width, dtype=torch.bfloat16, device=device)
        self.dbias, self.dgain = torch.empty(words, device=device), torch.empty(width, device=device)
        self.grad = torch.empty_like(self.weights)
        self.grads = gk.GradList([self.dw, self.dbias, self.dgain], out=self.grad)
        self.norm, self.norms = torch.empty(1, device=device), torch.empty(3, device=device)
        self.pairs = (torch.empty(self.weights.numel(), dtype=torch.int32, device=device), torch.empty_like(self.weights),
                      torch.zeros(1, dtype=torch.int64, device=device))

    def parts(self):
        w, bias, gain = torch.split(self.weights, [self.words * self.width, self.words, self.width])
        return w.view(self.words, self.width).bfloat16(), bias, gain

    def logits(self, h):
        w, bias, gain = self.parts()
        return (h * gain).bfloat16() @ w.t() + bias.bfloat16()

    def backward(self, h, dz):
        """The gradients of all weights from that of the logits, into the tensors that the GradList knows."""
        w, _, gain = self.parts()
        torch.mm(dz.t(), (h * gain).bfloat16(), out=self.dw)
        torch.sum(dz, 0, dtype=torch.float32, out=self.dbias)
        torch.sum((dz @ w).float() * h, 0, out=self.dgain)

    def step(self, rate: float, limit: float, keep: int):
        gk.gk_grad_norm(self.grads, self.norm, norms_out=self.norms)
        gk.gk_grad_clip(self.grads, limit, norm_in=self.norm)
        idx, val, nnz = self.pairs
        gk.gk_sparsify(self.grad, self.residual, keep, idx, val, nnz)
        gk.gk_apply_gathered(self.weights, idx, val, nnz, self.weights.numel(), -rate)


def loss_gradient(logits, token, advantage, bonus: float, out, keep: dict):
    """Gradient at the logits of the mean over rows of -advantage log p(token) - bonus entropy; rows whose token
    is negative are left out.  keep: buffers for what gk_vocab_logprob writes, which stay readable."""
    rows = max(1, int((token >= 0).sum()))
    gk.gk_vocab_logprob(logits, token, logp_out=keep["logp"], rank_out=keep["rank"], entropy_out=keep["entropy"],
                        lse_out=keep["lse"], idx_out=keep["idx"], val_out=keep["val"])
    gk.gk_vocab_logprob_grad(logits, token, keep["lse"], out, logp_grad=advantage * (-1.0 / rows), entropy=keep["entropy"],
                             entropy_grad=torch.full_like(keep["entropy"], -bonus / rows))
    return -(advantage * keep["logp"]).sum() / rows - bonus * keep["entropy"].sum() / rows


def buffers(rows: int, k: int, device):
    f = lambda *s: torch.empty(*s, device=device)  # noqa: E731
    i = lambda *s: torch.empty(*s, dtype=torch.int32, device=device)  # noqa: E731
    return {"logp": f(rows), "rank": i(rows), "entropy": f(rows), "lse": f(rows), "idx": i(rows, k), "val": f(rows, k)}


def train(steps: int = 60, rows: int = 512, width: int = 64, words: int = 1003, k: int = 5, density: float = 0.05,
          rate: float = 300.0, limit: float = 0.05, bonus: float = 0.003, seed: int = 0):
    """Returns (mean reward, mean entropy, norm of the gradients) of each step.  A row's hidden state names one word;
    sampling that word, or one of the next four, is rewarded."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    policy, keep = Policy(words, width, dev), buffers(rows, k, dev)
    states = torch.randn(words, width, generator=gen, device=dev) / width ** 0.5
    number = max(1, int(density * policy.weights.numel()))
    baseline, log = 0.0, []
    for _ in range(steps):
        goal = torch.randint(0, words // 20, (rows,), generator=gen, device=dev)
        h = states[goal]
        logits = policy.logits(h)
        noise = -torch.log(-torch.log(torch.rand(rows, words, generator=gen, device=dev).clamp_(1e-20, 1 - 1e-7)))
        token = (logits.float() + noise).argmax(1)
        reward = ((token - goal >= 0) & (token - goal < 5)).float()
        dz = torch.empty_like(logits)
        loss_gradient(logits, token, reward - baseline, bonus, dz, keep)
        policy.backward(h, dz)
        policy.step(rate, limit, number)
        baseline = 0.9 * baseline + 0.1 * float(reward.mean())
        log.append((float(reward.mean()), float(keep["entropy"].mean()), float(policy.norm)))
    return log


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    for i, (reward, entropy, norm) in enumerate(train(ap.parse_args().steps)):
        if i % 10 == 0:
            print(f"step {i:3d}  reward {reward:.4f}  entropy {entropy:.3f}  norm {norm:.4f}")


if __name__ == "__main__":
    main()
