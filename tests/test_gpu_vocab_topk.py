"""gk_vocab_topk against a stable sort in 64 bits: the pairs are exact, the log-sum-exp is within the
rounding of its sum (each term and the running sum are off by a few 2^-24 of themselves: 2^-19
relative to the sum covers it, plus 2^-21 of the result's magnitude)."""
import math

import pytest
import torch

from paper_1911_08772_b200 import binding as gk
from vocab_util import topk_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


def check(z, k, T=1.0, view=None):
    """z: CPU tensor (n, V); view: the device tensor the call reads (default: z's copy)."""
    n, V = z.shape
    view = z.to(DEV) if view is None else view
    idx = torch.full((n * k + 5,), -7, dtype=torch.int32, device=DEV)
    val = torch.full((n * k + 5,), -7.0, device=DEV)
    lse = torch.full((n + 5,), -7.0, device=DEV)
    gk.gk_vocab_topk(view, k, idx[:n * k].view(n, k), val[:n * k].view(n, k), lse_out=lse[:n], temperature=T)
    torch.cuda.synchronize()
    assert bool((idx[n * k:] == -7).all()) and bool((val[n * k:] == -7).all()) and bool((lse[n:] == -7).all())
    want = topk_reference(z, k)
    got = idx[:n * k].view(n, k).cpu().long()
    assert torch.equal(got, want)
    gv, wv = val[:n * k].view(n, k).cpu(), torch.gather(z.float(), 1, want)
    nan = torch.isnan(wv)
    assert torch.equal(torch.isnan(gv), nan)
    assert torch.equal(gv[~nan].view(torch.int32), wv[~nan].view(torch.int32))
    # the definition, with an infinite logit's row infinite and a NaN's NaN
    ref = torch.logsumexp(z.double() / T, 1)
    ref = torch.where(torch.isnan(z).any(1), torch.full_like(ref, math.nan), ref)
    gl = lse[:n].cpu().double()
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isnan(gl), torch.isnan(ref))
    assert torch.equal(gl[~fin & ~torch.isnan(ref)], ref[~fin & ~torch.isnan(ref)])
    assert bool(((gl - ref).abs()[fin] <= 2.0 ** -19 + 2.0 ** -21 * ref.abs()[fin]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (3, 2, 2), (1, 7, 3), (5, 33, 33), (4, 1000, 1), (3, 1024, 1024), (2, 4097, 64),
                                   (7, 10000, 100), (3, 32000, 1000), (2, 50001, 20), (1, 200003, 128), (300, 515, 9)])
def test_random_rows(n, V, k, dtype):
    gen = torch.Generator().manual_seed(n + V + k)
    check((torch.randn(n, V, generator=gen) * 3).to(dtype), k, T=1.0 if k % 2 else 1.7)


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_go_to_the_lower_index(dtype):
    gen = torch.Generator().manual_seed(3)
    for levels in (1, 2, 5):
        for V, k in ((700, 50), (20000, 600), (40000, 3)):
            check(torch.randint(0, levels, (3, V), generator=gen).to(dtype), k)
            check(-torch.randint(0, levels, (3, V), generator=gen).to(dtype) * 0.5, k)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_rows_infinities_and_nan(dtype):
    gen = torch.Generator().manual_seed(4)
    for V in (60, 3000, 30000):
        z = (torch.randn(8, V, generator=gen) * 2).to(dtype)
        z[0] = -math.inf                                   # nothing left
        z[1, 5:] = -math.inf                               # fewer than k left
        z[2, torch.rand(V, generator=gen) < 0.9] = -math.inf
        z[3] = torch.finfo(dtype).min                      # the type's lowest value
        z[4, 11] = math.inf
        z[5, 13] = math.nan
        z[6, ::2] = 0.0
        z[6, 1::2] = -0.0
        z[7, :40] = torch.finfo(dtype).max
        check(z, 33)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("order", ["ascending", "descending", "one_block"])
def test_rows_in_an_order(order, dtype):
    """The largest last, first, or all within a short stretch."""
    V = 30011
    z = torch.linspace(-9, 9, V).repeat(2, 1)
    if order == "descending":
        z = z.flip(1).contiguous()
    if order == "one_block":
        z = torch.zeros(2, V)
        z[:, 17000:17800] = torch.randn(2, 800, generator=torch.Generator().manual_seed(1)).abs() + 1
    check(z.to(dtype), 500)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 5)])
def test_row_strides_and_unaligned_rows(pad, shift, dtype):
    gen = torch.Generator().manual_seed(6)
    n, V = 5, 5003
    z = (torch.randn(n, V, generator=gen) * 2).to(dtype)
    store = torch.full((n * (V + pad) + shift,), 1e4, dtype=dtype, device=DEV)
    view = store[shift:].view(n, V + pad)[:, :V]
    view.copy_(z)
    check(z, 40, view=view)


def test_offsets_past_32_bits():
    n, V, k = 17000, 130001, 9          # 2.2e9 logits
    gen = torch.Generator(device=DEV).manual_seed(7)
    z = torch.empty(n, V, dtype=torch.bfloat16, device=DEV)
    for a in range(0, n, 1000):
        z[a:a + 1000] = torch.randn(1000, V, generator=gen, device=DEV).bfloat16()
    idx, val, lse = torch.empty(n, k, dtype=torch.int32, device=DEV), torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    gk.gk_vocab_topk(z, k, idx, val, lse_out=lse)
    for a in (0, 8000, n - 50):
        rows = z[a:a + 50]
        want = topk_reference(rows.cpu(), k)
        assert torch.equal(idx[a:a + 50].cpu().long(), want)
        assert torch.equal(val[a:a + 50].cpu(), torch.gather(rows.cpu().float(), 1, want))
        ref = torch.logsumexp(rows.double(), 1)
        assert bool(((lse[a:a + 50].double() - ref).abs() <= 2.0 ** -19 + 2.0 ** -21 * ref.abs()).all())


def test_without_log_sum_exp_and_without_rows():
    z = torch.randn(3, 500, device=DEV)
    idx, val = torch.empty(3, 4, dtype=torch.int32, device=DEV), torch.empty(3, 4, device=DEV)
    gk.gk_vocab_topk(z, 4, idx, val)
    assert torch.equal(idx.cpu().long(), topk_reference(z.cpu(), 4))
    gk.gk_vocab_topk(z[:0], 4, idx[:0], val[:0])


def test_refusals():
    z = torch.zeros(2, 50, device=DEV)
    idx, val = torch.empty(2, 4, dtype=torch.int32, device=DEV), torch.empty(2, 4, device=DEV)
    big = lambda k: (torch.empty(2, k, dtype=torch.int32, device=DEV), torch.empty(2, k, device=DEV))  # noqa: E731
    for args, kw in (((z.double(), 4, idx, val), {}), ((z.cpu(), 4, idx, val), {}), ((z, 3, idx, val), {}), ((z, 0, *big(0)), {}),
                     ((z, 51, *big(51)), {}), ((z, 4, idx.long(), val), {}), ((z, 4, idx, val), {"temperature": 0.0}),
                     ((z.t(), 4, idx, val), {}), ((z[0], 4, idx, val), {}), ((z, 4, idx, val), {"lse_out": torch.empty(3, device=DEV)}),
                     ((torch.zeros(2, 5000, device=DEV), 1025, *big(1025)), {})):
        with pytest.raises(gk.GkError):
            gk.gk_vocab_topk(*args, **kw)
