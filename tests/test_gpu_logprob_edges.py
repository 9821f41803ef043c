"""Calls of gk_vocab_logprob, gk_vocab_logprob_grad, gk_grad_norm and gk_grad_clip that the documentation allows and
ordinary use seldom makes: the longest rows, many rows, the same call again, several threads and streams."""
import math
import threading

import pytest
import torch

from grad_util import NORM_TOL, check_clipped, norms64, tensors
from logprob_util import bounds, close, grad_reference, logp_tol, reference
from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


def test_the_longest_row():
    V = 2 ** 31 - 1
    z = torch.zeros(1, V, dtype=BF16, device=DEV)
    planted = [5, V - 1, 2 ** 30 + 7]
    z[0, planted] = torch.tensor([30.0, 29.0, 28.0], dtype=BF16, device=DEV)
    token = torch.tensor([[2 ** 30 + 7, V - 1, 77]], device=DEV)
    logp, val = torch.empty(1, 3, device=DEV), torch.empty(1, 5, device=DEV)
    rank, idx = torch.empty(1, dtype=torch.int32, device=DEV), torch.empty(1, 5, dtype=torch.int32, device=DEV)
    lse, entropy = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    gk.gk_vocab_logprob(z, token, logp_out=logp, rank_out=rank, entropy_out=entropy, lse_out=lse, idx_out=idx, val_out=val)
    assert idx[0].tolist() == [5, V - 1, 2 ** 30 + 7, 0, 1] and int(rank) == 2
    # 2^20 equal terms a thread are exact in fp32 pairs; the rest as for ordinary rows
    total = (V - 3) + sum(math.exp(x) for x in (30, 29, 28))
    want = math.log(total)
    assert abs(float(lse) - want) <= 2e-5
    for got, x in zip(logp[0].tolist(), (28, 29, 0)):
        assert abs(got - (x - want)) <= 3e-5
    ent = (V - 3) / total * want - sum(math.exp(x) / total * (x - want) for x in (30, 29, 28))
    assert abs(float(entropy) - ent) <= 2e-5 * (1 + ent)
    gk.gk_vocab_logprob_grad(z, token, lse, z, logp_grad=torch.ones(1, 3, device=DEV))
    for i, one in ((5, 0), (V - 1, 1), (2 ** 30 + 7, 1), (77, 1), (78, 0), (V - 2, 0)):
        x = {5: 30.0, V - 1: 29.0, 2 ** 30 + 7: 28.0}.get(i, 0.0)
        true = one - 3 * math.exp(x - want)
        assert abs(float(z[0, i]) - true) <= 2.0 ** -8 * abs(true) + 1e-4 * math.exp(x - want)


@pytest.mark.parametrize("V,dtype", [(3, F32), (17, BF16), (1003, F16)])
def test_more_rows_than_a_grid_has_in_one_direction(V, dtype):
    n = 140001
    gen = torch.Generator().manual_seed(V)
    z = (torch.randn(n, V, generator=gen) * 2).to(dtype)
    token = torch.randint(-1, V, (n, 1), generator=gen)
    k = min(V, 2)
    lse, logp, entropy, val = torch.empty(n, device=DEV), torch.empty(n, 1, device=DEV), torch.empty(n, device=DEV), torch.empty(n, k, device=DEV)
    idx, dz = torch.empty(n, k, dtype=torch.int32, device=DEV), torch.empty(n, V, dtype=dtype, device=DEV)
    a = torch.randn(n, 1, generator=gen)
    gk.gk_vocab_logprob(z.to(DEV), token.to(DEV), logp_out=logp, entropy_out=entropy, lse_out=lse, idx_out=idx, val_out=val)
    gk.gk_vocab_logprob_grad(z.to(DEV), token.to(DEV), lse, dz, logp_grad=a.to(DEV))
    some = torch.cat([torch.arange(300), torch.arange(65500, 65600), torch.arange(n - 300, n)])
    ref = reference(z[some], token[some], 1.0, k)
    assert close(lse[some.to(DEV)], ref["lse"], bounds(z[some], ref, 1.0)["lse"])
    assert close(logp[some.to(DEV)], ref["logp"], logp_tol(ref["logp"]))
    assert torch.equal(idx[some.to(DEV)].cpu().long(), ref["idx"])
    want, tol = grad_reference(z[some], token[some], 1.0, lse[some.to(DEV)].cpu(), entropy[some.to(DEV)].cpu(), a[some], None, None)
    u = torch.finfo(dtype).eps / 2
    assert close(dz[some.to(DEV)], want, tol + u * (want.abs() + tol) + (2.0 ** -25 if dtype == F16 else 2.0 ** -126))


@pytest.mark.parametrize("n,V,k,dtype", [(37, 8000, 7, BF16), (300, 515, 9, F32), (1, 50001, 20, F32), (2000, 6000, 100, F16), (5, 128000, 128, BF16),
                                         (700, 128000, 20, BF16)])
def test_the_same_call_gives_the_same_bits(n, V, k, dtype):
    gen = torch.Generator(device=DEV).manual_seed(n)
    z = (torch.randn(n, V, generator=gen, device=DEV) * 3).to(dtype)
    token = torch.randint(0, V, (n, 2), generator=gen, device=DEV)
    first = None
    for _ in range(5):
        f, i = [torch.empty(n, device=DEV) for _ in range(2)], [torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, k, dtype=torch.int32, device=DEV)]
        logp, val = torch.empty(n, 2, device=DEV), torch.empty(n, k, device=DEV)
        gk.gk_vocab_logprob(z, token, logp_out=logp, rank_out=i[0], entropy_out=f[0], lse_out=f[1], idx_out=i[1], val_out=val)
        out = f + i + [logp, val]
        first = first or out
        assert all(torch.equal(x, y) for x, y in zip(first, out))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("k", [3, 90])
def test_few_tokens_allowed(dtype, k):
    """Structured output: all but a few logits are masked, by -inf or by the type's lowest value; the token may be a
    masked one."""
    gen = torch.Generator().manual_seed(k)
    for V, n in ((700, 40), (33000, 6), (128000, 2)):
        for mask in (-math.inf, torch.finfo(dtype).min):
            z = torch.full((n, V), mask)
            allowed = torch.randint(0, V, (n, 5), generator=gen)
            z.scatter_(1, allowed, torch.randn(n, 5, generator=gen) * 4)
            z = z.to(dtype)
            token = allowed[:, :1].clone()
            token[0] = V - 1
            lse, entropy, rank = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, dtype=torch.int32, device=DEV)
            logp, val, idx = torch.empty(n, 1, device=DEV), torch.empty(n, k, device=DEV), torch.empty(n, k, dtype=torch.int32, device=DEV)
            gk.gk_vocab_logprob(z.to(DEV), token.to(DEV), logp_out=logp, rank_out=rank, entropy_out=entropy, lse_out=lse, idx_out=idx, val_out=val)
            ref = reference(z, token, 1.0, k)
            tol = bounds(torch.where(z < -1e4, torch.zeros_like(z), z), ref, 1.0)
            assert close(lse, ref["lse"], tol["lse"]) and close(entropy, ref["entropy"], tol["entropy"])
            assert torch.equal(rank.cpu().long(), ref["rank"]) and torch.equal(idx.cpu().long(), ref["idx"])
            fine = ref["val"] > -1e4
            assert close(torch.where(fine.to(DEV), val, 0.0), torch.where(fine, ref["val"], 0.0), logp_tol(torch.where(fine, ref["val"], 0.0)))


def test_clipping_by_several_threads_on_one_stream_and_on_their_own():
    work = []
    for seed, t in enumerate((F32, BF16, F16, F32)):
        grads = tensors([50001 * (seed + 1), 77, 30000], [t], seed=seed)
        n = sum(g.numel() for g in grads)
        work.append((grads, 0.4 * float(norms64(grads).square().sum().sqrt()), torch.empty(n, device=DEV), torch.empty(1, device=DEV)))
    torch.cuda.synchronize()
    for own in (False, True):
        failed = []
        gate = threading.Barrier(len(work))

        def body(item):
            grads, limit, out, norm = item
            try:
                stream = torch.cuda.Stream() if own else torch.cuda.default_stream()
                gate.wait()
                with torch.cuda.stream(stream):
                    for _ in range(20):
                        gk.gk_grad_clip(grads, limit, out=out, norm_out=norm)
                        gk.gk_grad_norm(grads, norm)
                    stream.synchronize()
            except Exception as e:      # noqa: BLE001
                failed.append(e)

        threads = [threading.Thread(target=body, args=(w,)) for w in work]
        [t.start() for t in threads]
        [t.join() for t in threads]
        assert not failed, failed
        for grads, limit, out, norm in work:
            total = float(norms64(grads).square().sum().sqrt())
            assert abs(float(norm) - total) <= NORM_TOL * total
            check_clipped(grads, torch.split(out, [g.numel() for g in grads]), limit)


def test_norm_and_clipping_after_one_another_without_waiting():
    """A norm's tensors are the next call's outputs: the calls of a stream see one another's results."""
    grads = tensors([200_003, 4099, 5], [F32])
    before = [g.clone() for g in grads]
    norm, norms = torch.empty(1, device=DEV), torch.empty(3, device=DEV)
    limit = 0.5 * float(norms64(grads).square().sum().sqrt())
    for i in range(10):
        gk.gk_grad_norm(grads, norm, norms_out=norms)
        gk.gk_grad_clip(grads, limit * 0.5 ** i, norm_in=norm)
    # each call scales by about a half
    total = float(norms64(before).square().sum().sqrt())
    assert abs(float(norm) - total * 0.5 ** 9) <= 12 * NORM_TOL * total
    for g, b in zip(grads, before):
        assert float((g.double() - b.double() * 2.0 ** -10).abs().max()) <= 12 * 11 * 2.0 ** -24 * float(b.abs().max()) * 2.0 ** -10


def test_as_many_tensors_as_are_allowed():
    n = 65536
    flat = torch.randn(2 * n, device=DEV)
    grads = list(torch.split(flat, 2))
    norm, norms = torch.empty(1, device=DEV), torch.empty(n, device=DEV)
    gk.gk_grad_norm(grads, norm, norms_out=norms)
    want = flat.double().view(n, 2).norm(dim=1)
    assert bool(((norms.double() - want).abs() <= NORM_TOL * want).all())
    assert abs(float(norm) - float(flat.double().norm())) <= NORM_TOL * float(flat.double().norm())
    out = torch.empty_like(flat)
    gk.gk_grad_clip(grads, 1.0, out=out, norm_out=norm)
    check_clipped([flat], [out], 1.0)
    with pytest.raises(gk.GkError):
        gk.gk_grad_norm(grads + [flat[:1]], norm)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gradients_between_the_rows_of_their_logits(dtype):
    """Two halves of one buffer's rows; rows that meet are refused."""
    n, V, gap = 9, 1003, 5
    gen = torch.Generator().manual_seed(4)
    both = torch.full((n, 2 * V + gap), 7.0, dtype=dtype, device=DEV)
    z, dz = both[:, :V], both[:, V + 2:2 * V + 2]
    z.copy_((torch.randn(n, V, generator=gen) * 2).to(dtype))
    token, a = torch.randint(0, V, (n, 1), generator=gen), torch.randn(n, 1, generator=gen)
    lse, entropy = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    gk.gk_vocab_logprob(z, token.to(DEV), lse_out=lse, entropy_out=entropy)
    kept = z.cpu()
    gk.gk_vocab_logprob_grad(z, token.to(DEV), lse, dz, logp_grad=a.to(DEV))
    want, tol = grad_reference(kept, token, 1.0, lse.cpu(), entropy.cpu(), a, None, None)
    u = torch.finfo(dtype).eps / 2
    assert close(dz, want, tol + u * (want.abs() + tol) + (2.0 ** -25 if dtype == F16 else 2.0 ** -126))
    assert torch.equal(z.cpu(), kept)
    assert bool((both[:, V:V + 2] == 7).all()) and bool((both[:, 2 * V + 2:] == 7).all())
    for bad in (both[:, V - 1:2 * V - 1], both.as_strided((n - 1, V), (2 * V + gap + 1, 1), V + 2)):
        with pytest.raises(gk.GkError):
            gk.gk_vocab_logprob_grad(z[:len(bad)], token[:len(bad)].to(DEV), lse[:len(bad)], bad, logp_grad=a[:len(bad)].to(DEV))
    # the logits behind their gradients
    gk.gk_vocab_logprob_grad(dz, token.to(DEV), lse, z, logp_grad=a.to(DEV))
