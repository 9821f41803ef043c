"""gk_vocab_logprob on rows masked with ordinary finite values, and on rows whose largest logit is far from zero."""
import math

import pytest
import torch

from logprob_util import S_TOL, U, bounds, close, grad_reference, logp_tol, reference
from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
PATTERNS = ["few", "few_in_the_first_words", "one_stretch", "half", "none"]
# rows of one CTA of 64, 128 and 256 threads; of several CTAs
LAUNCHES = [(160, 700), (700, 10000), (160, 33000), (20, 8001), (20, 33000), (2, 128000)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


def row(V, pattern, mask, gen):
    """(logits, which of them are masked)"""
    on = torch.zeros(V, dtype=torch.bool)
    if pattern == "few":
        on[torch.randint(V // 8, V // 4, (5,), generator=gen)] = True
    elif pattern == "few_in_the_first_words":
        on[:5] = True
    elif pattern == "one_stretch":
        on[V // 2:V // 2 + V // 7] = True
    elif pattern == "half":
        on = torch.rand(V, generator=gen) < 0.5
    z = torch.where(on, torch.randn(V, generator=gen) * 3, torch.full((), mask))
    return z, ~on


def compare(z, T, k, token, big, full):
    """Calls the operator on the rows of z, repeated to `full` rows, and compares the first of each with the
    definition.  big: |z| that the log-sum-exp's rounding is of (rows without a maximum near zero)."""
    n, V = z.shape
    again = -(-full // n)
    zd, td = z.to(DEV).repeat(again, 1)[:max(full, n)], token.to(DEV).repeat(again, 1)[:max(full, n)]
    rows, m = zd.shape[0], token.shape[1]
    logp, rank, entropy, lse = torch.empty(rows, m, device=DEV), torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    idx, val = torch.empty(rows, k, dtype=torch.int32, device=DEV), torch.empty(rows, k, device=DEV)
    gk.gk_vocab_logprob(zd, td, temperature=T, logp_out=logp, rank_out=rank, entropy_out=entropy, lse_out=lse, idx_out=idx, val_out=val)
    plain = torch.empty(rows, device=DEV)
    gk.gk_vocab_logprob(zd, td, temperature=T, lse_out=plain)
    ref = reference(z, token, T, k)
    tol = bounds(big, ref, T)
    inf32 = lambda x: x.float().double()      # noqa: E731  what fp32 has no number for is an infinity
    for at in range(0, rows, n):      # (a row's elements lie otherwise in its words where V is odd)
        here, own = slice(at, min(rows, at + n)), slice(0, min(rows, at + n) - at)
        assert close(lse[here], inf32(ref["lse"][own]), tol["lse"][own]) and close(plain[here], inf32(ref["lse"][own]), tol["lse"][own])
        assert close(entropy[here], ref["entropy"][own], tol["entropy"][own])
        assert close(logp[here], inf32(ref["logp"][own]), logp_tol(ref["logp"][own]))
        assert close(val[here], inf32(ref["val"][own]), logp_tol(ref["val"][own]))
        assert torch.equal(rank[here].cpu().long(), ref["rank"][own]) and torch.equal(idx[here].cpu().long(), ref["idx"][own])
    return lse[:n], entropy[:n]


def masks(dtype):
    if dtype == F16:
        return [-1e3, -1e4, -30000.0, torch.finfo(F16).min]
    return [-1e4, -1e5, -1e6, -1e7, -1e8, -1e9, -1e10, -1e12, -1e20, -1e30, torch.finfo(dtype).min]


@pytest.mark.parametrize("n,V", LAUNCHES)
@pytest.mark.parametrize("dtype,T", [(F32, 1.0), (F32, 2.0), (F32, 1.5), (F32, 0.05), (BF16, 1.0), (BF16, 2.0), (BF16, 1.5), (BF16, 0.5),
                                     (F16, 1.0), (F16, 0.09), (F16, 0.05), (F16, 0.02), (F16, 30.0), (F32, 1000.0), (BF16, 1e5), (F32, 1e26)])
def test_rows_masked_with_finite_values(n, V, dtype, T):
    """Bounds: a masked logit's probability is nothing beside an allowed one's at these temperatures or is counted by
    the definition as well; the log-sum-exp's rounding is that of the largest logit, which is an allowed one's where
    there is one."""
    T = float(torch.tensor(T, dtype=F32))
    gen = torch.Generator().manual_seed(V + n)
    some = masks(dtype)
    if n == 2:
        some = some[-6::2]
    z, big, token = [], [], []
    for i, mask in enumerate(some):
        for pattern in PATTERNS if n > 2 else PATTERNS[:1]:
            x, masked = row(V, pattern, mask, gen)
            x = x.to(dtype)
            # (at temperatures that leave masked logits some weight, and where nothing is allowed, they count)
            count = pattern == "none" or abs(mask) / T < 1e4
            z.append(x)
            big.append(x if count else x.masked_fill(masked, 0.0))
            allowed = torch.nonzero(~masked)[:, 0]
            token.append(torch.tensor([int(allowed[0]) if len(allowed) else 3, V - 1]))
    z, big, token = torch.stack(z), torch.stack(big), torch.stack(token)
    for at in range(0, len(z), 20 if n > 2 else 2):
        to = at + (20 if n > 2 else 2)
        lse, entropy = compare(z[at:to], T, 7, token[at:to], big[at:to], n)
        rows = len(z[at:to])
        a, b = torch.randn(rows, 2, generator=gen), torch.randn(rows, generator=gen)
        dz = torch.empty(rows, V, dtype=dtype, device=DEV)
        gk.gk_vocab_logprob_grad(z[at:to].to(DEV), token[at:to].to(DEV), lse.contiguous(), dz, logp_grad=a.to(DEV), entropy=entropy.contiguous(),
                                 entropy_grad=b.to(DEV), temperature=T)
        want, tol = grad_reference(z[at:to], token[at:to], T, lse.cpu(), entropy.cpu(), a, b, None)
        u = torch.finfo(dtype).eps / 2
        # powers below fp32's normal range are zero: log p is above -104 for them; fp16's smallest half step
        flushed = 2.0 ** -126 * (1 + (a.abs().sum(1) + b.abs() * (entropy.cpu() + 104)).double() / T)[:, None] + (2.0 ** -25 if dtype == F16 else 0.0)
        # (rows without an allowed logit: log p is what the rounding of lse leaves, in both)
        sure = lse.cpu().abs() < 1e6
        assert close(dz[sure.to(DEV)], want[sure], (tol + u * (want.abs() + tol) + flushed)[sure])


@pytest.mark.parametrize("n,V", LAUNCHES[:5])
@pytest.mark.parametrize("power", [20, 21])
@pytest.mark.parametrize("sign", [-1, 1])
def test_rows_whose_exponents_are_next_to_a_power_of_two(n, V, power, sign):
    """z log2(e) about 2^20 and 2^21: neither the start of a thread's sums nor the maximum shows in an entropy."""
    gen = torch.Generator().manual_seed(power)
    centre = sign * 2.0 ** power * math.log(2)
    z = []
    for i in range(12):
        base = centre + (i - 6) * 1.7
        x = base + torch.randn(V, generator=gen)
        if i % 3 == 1:
            x = x.sort().values
        if i % 3 == 2:
            x += torch.linspace(-40, 4, V)
        z.append(x)
    z = torch.stack(z)
    compare(z, 1.0, 3, torch.randint(0, V, (12, 1), generator=gen), z, n)


@pytest.mark.parametrize("n,V", LAUNCHES)
def test_what_a_mask_is_has_no_say(n, V):
    """A mask's value, from -1e5 on, has no say in log-sum-exp, entropy and log probability: two results differ by what
    each may be off by."""
    gen = torch.Generator().manual_seed(5)
    on = torch.rand(n, V, generator=gen) < 4.0 / V
    on[:, V // 3] = True
    base = torch.randn(n, V, generator=gen) * 2
    token = torch.full((n, 1), V // 3, device=DEV)
    first = None
    for mask in (-math.inf, -1e5, -1e6, -1e7, -1e8, -1e9, -1e10, -1e15, -1e25, -3e38):
        z = torch.where(on, base, torch.full((), mask)).to(DEV)
        out = [torch.empty(n, device=DEV) for _ in range(3)]
        gk.gk_vocab_logprob(z, token, logp_out=out[0], lse_out=out[1], entropy_out=out[2])
        first = first or out
        for x, y in zip(first, out):
            assert bool(((x - y).abs() <= 2 * (S_TOL + 6 * U) * (1 + 2 * x.abs())).all()), mask
