"""The example of a head that learns from rewards: it runs, and its gradient is the one that automatic
differentiation gives for the same loss in 64 bits."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_1911_08772_b200 import binding as gk, build
    build.build()
    gk.load()
    gk.gk_set_capacity(0)
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import policy_head
    finally:
        sys.path.pop(0)
    return policy_head


def test_it_runs(example):
    log = example.train(steps=6, rows=96, width=32, words=403)
    assert len(log) == 6 and all(math.isfinite(x) for row in log for x in row)
    # a policy of zeros: every word alike
    assert abs(log[0][1] - math.log(403)) <= 1e-3 and log[0][2] > 0


def test_the_gradient_from_the_loss_to_the_sparsifiers_vector(example):
    from paper_1911_08772_b200 import binding as gk
    dev, rows, width, words, bonus = torch.device("cuda"), 60, 32, 203, 0.01
    gen = torch.Generator(device=dev).manual_seed(4)
    policy, keep = example.Policy(words, width, dev), example.buffers(rows, 3, dev)
    policy.weights[:words * width] = torch.randn(words * width, generator=gen, device=dev).bfloat16().float()
    policy.weights[words * width:-width] = torch.randn(words, generator=gen, device=dev).bfloat16().float()
    h = torch.randn(rows, width, generator=gen, device=dev).bfloat16().float()
    token = torch.randint(0, words, (rows,), generator=gen, device=dev)
    token[::7] = -1
    advantage = torch.randn(rows, generator=gen, device=dev)
    logits = policy.logits(h)
    dz = torch.empty_like(logits)
    loss = example.loss_gradient(logits, token, advantage, bonus, dz, keep)

    z = logits.double().requires_grad_()
    on = token >= 0
    logp = torch.log_softmax(z, 1)
    entropy = -(logp.exp() * logp).sum(1)
    want = (-(advantage.double() * logp.gather(1, token.clamp(min=0)[:, None])[:, 0]) - bonus * entropy)[on].sum() / int(on.sum())
    want.backward()
    # every term of the mean is off by at most 2^-16 of itself and one (see the bounds of gk_vocab_logprob's tests)
    assert abs(float(loss) - float(want.detach())) <= 2.0 ** -16 * (1 + float(advantage.abs().mean()) * 20)
    # p in fp32 and the rounding to bf16, half a step of 2^-7
    off = (dz.double() - z.grad).abs()
    assert bool((off <= z.grad.abs() * (2.0 ** -8 + 2.0 ** -14) + 2.0 ** -20 * z.grad.abs().max()).all())

    policy.backward(h, dz)
    limit = 0.5 * float(torch.cat([policy.dw.double().view(-1), policy.dbias.double(), policy.dgain.double()]).norm())
    gk.gk_grad_norm(policy.grads, policy.norm, norms_out=policy.norms)
    gk.gk_grad_clip(policy.grads, limit, norm_in=policy.norm)
    flat = torch.cat([policy.dw.double().view(-1), policy.dbias.double(), policy.dgain.double()])
    assert abs(float(policy.norm) - 2 * limit) <= 2.0 ** -20 * limit
    assert float((policy.grad.double() - flat / 2).abs().max()) <= 2.0 ** -20 * float(flat.abs().max())

    before, residual = policy.weights.clone(), policy.residual.clone()
    policy.step(1.0, limit, 500)
    idx, val, nnz = policy.pairs
    n = int(nnz)
    # what was sent and what was kept are the clipped gradient, and the weights moved by what was sent
    sent = torch.zeros_like(before)
    sent[idx[:n].long()] = val[:n]
    assert torch.equal(sent + policy.residual, policy.grad + residual)
    assert torch.equal(policy.weights, before - sent)
