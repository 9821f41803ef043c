"""Gradients for the tests of gk_grad_norm and gk_grad_clip, and the bounds that they are held to.

Bounds, from the arithmetic (relative):
  * a norm: up to 64 squares are added in fp32 by two chains of 32 fused multiply-adds, each off by 2^-24 of its
    partial sum, and joined: 33 x 2^-24 of the sum at most, half of that of its root; fp64 adds nothing that shows;
    one rounding to fp32: 17.5 x 2^-24, and below fp32's normal range half of its smallest step, 2^-149;
  * a clipped value: the coefficient's error, which is the norm's before rounding and one rounding to fp32, and the
    product's rounding: 18.5 x 2^-24, then the output type's half step eps / 2, or half of its smallest step."""
from __future__ import annotations

import torch

NORM_TOL, NORM_STEP = 17.5 * 2.0 ** -24, 2.0 ** -149
CLIP_TOL = 18.5 * 2.0 ** -24
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def tensors(sizes, types, seed=0, scale=1e-2, shift=0, device="cuda:0"):
    """Gradients with scales of their own; shift: elements between an allocation's start and the tensor's."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = types[i % len(types)]
        store = torch.full((n + shift + 3,), 7.0, dtype=t, device=device)
        g = store[shift:shift + n]
        g.copy_((torch.randn(n, generator=gen) * scale * (1 + i % 7)).to(t))
        out.append(g)
    return out


def norms64(grads):
    return torch.stack([g.double().square().sum().sqrt() for g in grads]).cpu() if grads else torch.zeros(0, dtype=torch.float64)


def check_norms(grads, norm, norms=None):
    want = norms64(grads)
    total = float(want.square().sum().sqrt())
    assert abs(float(norm) - total) <= NORM_TOL * total + NORM_STEP
    if norms is not None:
        assert bool(((norms.cpu().double() - want).abs() <= NORM_TOL * want + NORM_STEP).all())


def check_clipped(before, out, max_norm, scale=1.0, norm=None):
    """before: the gradients as they were; out: what the call wrote."""
    total = float(norms64(before).square().sum().sqrt()) * abs(scale) if norm is None else norm
    c = scale * (max_norm / total if total > max_norm else 1.0)
    for g, o in zip(before, out):
        want = g.double() * c
        off = (o.double() - want).abs()
        u = torch.finfo(o.dtype).eps / 2
        assert bool((off <= CLIP_TOL * want.abs() + u * want.abs() * (1 + CLIP_TOL) + TINY[o.dtype]).all())
