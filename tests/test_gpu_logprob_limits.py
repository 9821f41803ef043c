"""gk_vocab_logprob and gk_vocab_logprob_grad at the ends of what they take."""
import math

import pytest
import torch

from logprob_util import U, bounds, close, grad_reference, logp_tol, reference
from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SMALLEST = {F32: 2.0 ** -126, BF16: 2.0 ** -126, F16: 2.0 ** -25}


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


def run(z, token, T, k=0):
    n, m = token.shape
    out = {"logp": torch.empty(n, m, device=DEV), "rank": torch.empty(n, dtype=torch.int32, device=DEV), "entropy": torch.empty(n, device=DEV),
           "lse": torch.empty(n, device=DEV)}
    if k:
        out["idx"], out["val"] = torch.empty(n, k, dtype=torch.int32, device=DEV), torch.empty(n, k, device=DEV)
    gk.gk_vocab_logprob(z.to(DEV), token.to(DEV), temperature=T, **{name + "_out": x for name, x in out.items()})
    return out


def near_zero(V, T, dtype, gen):
    """Rows whose largest logit is 0, the others a few T below it or far."""
    z = -torch.randn(6, V, generator=gen).abs().double() * 4 * T
    z[:, V // 2] = 0
    z[0] = 0
    z[2, torch.rand(V, generator=gen) < 0.5] = -math.inf
    z[3, 5:V // 2] = torch.finfo(dtype).min
    z[4, ::3] = -1.0
    z[5, :V // 2] = -math.inf
    return z.to(dtype)


@pytest.mark.parametrize("T", [1e-7, 1e-9, 1e-20, 1e-30, 1e-37])
@pytest.mark.parametrize("V", [60, 1003, 8192, 50001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_entropies_at_the_smallest_temperatures(T, V, dtype):
    T = float(torch.tensor(T, dtype=F32))
    gen = torch.Generator().manual_seed(V)
    z = near_zero(V, T, dtype, gen)
    token = torch.stack([torch.randint(0, V, (6,), generator=gen), torch.full((6,), V // 2)], 1)
    out, ref = run(z, token, T, 4), reference(z, token, T, 4)
    tol = bounds(torch.zeros_like(z), ref, T)
    assert close(out["lse"], ref["lse"], tol["lse"])
    assert close(out["entropy"], ref["entropy"], tol["entropy"])
    assert torch.equal(out["rank"].cpu().long(), ref["rank"]) and torch.equal(out["idx"].cpu().long(), ref["idx"])


@pytest.mark.parametrize("T", [1e-7, 1e-20, 1e-36])
def test_fp16_at_the_smallest_temperatures(T):
    """Logits that differ are infinitely far apart here, beside 2^-24."""
    z = torch.full((3, 1003), -2.0, dtype=F16)
    z[:, 700:704] = 0
    z[1, :700] = -math.inf
    z[2, :500] = torch.finfo(F16).min
    T = float(torch.tensor(T, dtype=F32))
    token = torch.tensor([[701], [702], [1]])
    out, ref = run(z, token, T), reference(z, token, T, 0)
    tol = bounds(torch.zeros_like(z), ref, T)
    assert close(out["lse"], ref["lse"], tol["lse"]) and close(out["entropy"], ref["entropy"], tol["entropy"])


@pytest.mark.parametrize("T", [3.3e-8, 1e-9, 1.1e-9, 1.3e-9, 7.7e-10, 3.3e-12])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_log_probabilities_below_the_range_of_fp32(T, dtype):
    """z / T beyond fp32 is an infinity of the logit's own sign, whatever that of the second part of 1 / T (which is
    negative but for 1e-9)."""
    V = 1003
    t = float(torch.tensor(T, dtype=F32))
    z = torch.zeros(4, V)
    z[0, 7:] = torch.finfo(dtype).min
    z[1, :900] = -1e38
    z[2] = torch.finfo(dtype).min
    z[3] = 3e38
    z = z.to(dtype)
    token = torch.tensor([[500, 3], [1, 999], [8, 9], [8, 9]])
    out, ref = run(z, token, t, 9), reference(z, token, t, 9)
    for name in ("logp", "val", "lse"):
        want = ref[name].float().double()
        assert close(out[name], want, logp_tol(want)), (name, t)
    assert close(out["entropy"], ref["entropy"], bounds(torch.zeros_like(z), ref, t)["entropy"])


@pytest.mark.parametrize("bits", [-1, 0x7fffffff, 0x7fc00000, -0x400000, 0x7f800001, -0x7fffff])
@pytest.mark.parametrize("n,V", [(1, 50001), (3, 128000), (2, 700), (300, 8001)])
def test_the_rank_of_a_token_whose_logit_is_nan(n, V, bits):
    """NaN counts as above +inf, whatever its bits; equal ones in order of increasing index."""
    z = torch.randn(n, V, generator=torch.Generator().manual_seed(V)).abs()
    z[:, 11] = math.inf
    z.view(torch.int32)[:, V - 9] = bits
    token = torch.full((n, 1), V - 9)
    out = run(z, token, 1.0, 2)
    assert bool((out["rank"] == 0).all()) and bool((out["idx"] == torch.tensor([V - 9, 11], device=DEV)).all())
    z.view(torch.int32)[:, V // 2] = 0x7fc00000
    out = run(z, token, 1.0, 2)
    assert bool((out["rank"] == 1).all()) and bool((out["idx"] == torch.tensor([V // 2, V - 9], device=DEV)).all())


def layouts(n, V, dtype):
    """(logits' rows, gradients' rows) as views: alike, at odd places, at other 16-byte boundaries, in place."""
    def view(pad, shift):
        return torch.full((n * (V + pad) + shift,), 7.0, dtype=dtype, device=DEV)[shift:].view(n, V + pad)[:, :V]
    yield view(0, 0), view(0, 0)
    yield view(5, 3), view(5, 3)
    yield view(0, 0), view(3, 1)
    z = view(1, 1)
    yield z, z


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("given", ["logp", "entropy", "lse", "all"])
def test_gradients_of_rows_without_a_log_sum_exp_are_nan_throughout(given, dtype):
    n, V = 4, 1003
    z = torch.randn(n, V, generator=torch.Generator().manual_seed(2)).to(dtype)
    z[1, 500], z[2, 3] = math.inf, math.nan
    z[:, 40:60] = -math.inf
    z[1:3, V - 1] = -math.inf
    token = torch.tensor([[1], [2], [3], [4]], device=DEV)
    ones = torch.ones(n, device=DEV)
    for view, out in layouts(n, V, dtype):
        view.copy_(z)
        lse, entropy = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        gk.gk_vocab_logprob(view, token, lse_out=lse, entropy_out=entropy)
        assert float(lse[1]) == math.inf and math.isnan(float(lse[2]))
        gk.gk_vocab_logprob_grad(view, token, lse, out, logp_grad=ones[:, None] if given in ("logp", "all") else None,
                                 entropy=entropy, entropy_grad=ones if given in ("entropy", "all") else None,
                                 lse_grad=ones if given in ("lse", "all") else None)
        assert torch.isnan(out).all(1).tolist() == [False, True, True, False]
        assert torch.isnan(out).any(1).tolist() == [False, True, True, False]
    # left out, they are zero
    token[1:3] = -100
    for view, out in layouts(n, V, dtype):
        view.copy_(z)
        gk.gk_vocab_logprob_grad(view, token, lse, out, logp_grad=ones[:, None])
        assert bool((out[1:3] == 0).all())


EXTREMES = [(1e5, 300.0), (3e37, 1e36), (2.0 ** -30, 1.0), (2.0 ** -66, 2.0 ** -66), (2.0 ** -66, 1.0), (2.0 ** -100, 1.0)]


@pytest.mark.parametrize("T,size", EXTREMES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_masked_logits_have_no_gradient(dtype, T, size):
    """Logits of -inf have no gradient, whatever T and the gradients given: at large T the type's lowest value has a
    probability, at small T factors of 1 / T go past fp32 beside a probability of zero."""
    n, V = 5, 1003
    gen = torch.Generator().manual_seed(3)
    z = torch.randn(n, V, generator=gen)
    if T < 1:
        # one logit at 8, in the others' words or at the row's end, the rest at 7 and below
        z = z.clamp(-7, 7)
        z[torch.arange(n), torch.tensor([0, 5, 500, V - 1, 77])] = 8.0
    z[:, 100:300] = -math.inf
    z[:, V - 3:V - 1] = -math.inf
    z[1:, 1] = -math.inf
    z = z.to(dtype)
    token = torch.tensor([[0], [5], [500], [V - 1], [200]])
    a, b = torch.randn(n, 1, generator=gen) * size, torch.randn(n, generator=gen) * size
    if dtype == F16 and T < 1:
        a, b = a * T, b * T      # in fp16's range
    T = float(torch.tensor(T, dtype=F32))
    ref = reference(z, token, T, 0)
    lse, entropy = ref["lse"].float(), ref["entropy"].float()
    if T < 1:
        assert torch.equal(lse.double(), ref["lse"])
    want, tol = grad_reference(z, token, T, lse, entropy, a, b, None)
    u = torch.finfo(dtype).eps / 2
    flushed = 2.0 ** -126 * (1 + (a.abs().sum(1) + b.abs() * (entropy + 104)).double() / T)[:, None]
    gone = (z == -math.inf).to(DEV)
    gone[torch.arange(n), token[:, 0]] = False
    for view, out in layouts(n, V, dtype):
        view.copy_(z)
        gk.gk_vocab_logprob_grad(view, token.to(DEV), lse.to(DEV), out, logp_grad=a.to(DEV), entropy=entropy.to(DEV), entropy_grad=b.to(DEV),
                                 temperature=T)
        assert bool((out[gone] == 0).all()), T
        fine = (want.abs() < torch.finfo(dtype).max)
        assert close(torch.where(fine.to(DEV), out, 0.0), torch.where(fine, want, 0.0), tol + u * (want.abs() + tol) + flushed + SMALLEST[dtype]), T


@pytest.mark.parametrize("T,size", [(1e31, 3e31), (1e34, 1e34), (1e36, 3e36), (1e38, 1e38), (3e38, 1e38)])
@pytest.mark.parametrize("n,V", [(160, 700), (5, 8001), (2, 128000), (160, 33000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_that_are_further_apart_than_fp32_reaches(dtype, n, V, T, size):
    """A mask of the lowest value under large logits, at temperatures that leave it a finite log probability."""
    T = float(torch.tensor(T, dtype=F32))
    gen = torch.Generator().manual_seed(V)
    z = torch.randn(12, V, generator=gen).clamp(-3, 3) * size
    z[:4, torch.rand(V, generator=gen) < 0.5] = torch.finfo(dtype).min
    z[4:8, V // 9:] = torch.finfo(dtype).min
    z[3] = torch.finfo(dtype).min
    z[2, V // 2], z[7, 3] = 3.3e38, 3.3e38
    z = z.to(dtype).repeat(-(-n // 12), 1)[:n] if n > 12 else z[[0, 2, 3, 5, 7]][:n].to(dtype)
    token = torch.randint(0, V, (n, 2), generator=gen)
    out, ref = run(z, token, T, 5), reference(z[:12], token[:12], T, 5)
    # (a difference whose ends are scaled first is rounded two times more, both of numbers below it)
    first = {name: x[:12] for name, x in out.items()}
    assert close(first["lse"], ref["lse"], bounds(z[:12], ref, T)["lse"])
    assert close(first["entropy"], ref["entropy"], bounds(z[:12], ref, T)["entropy"])
    for name in ("logp", "val"):
        assert close(first[name], ref[name], logp_tol(ref[name]) + 6 * U * ref[name].abs())
    assert torch.equal(first["rank"].cpu().long(), ref["rank"]) and torch.equal(first["idx"].cpu().long(), ref["idx"])
