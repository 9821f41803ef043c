"""gk_vocab_logprob and gk_vocab_logprob_grad against the definitions in 64 bits."""
import math

import pytest
import torch

from logprob_util import bounds, close, grad_reference, logp_tol, reference
from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


def padded(n, k, dtype=F32):
    """A (n, k) buffer with marked elements behind it, which the caller's check finds as they were."""
    store = torch.full((n * k + 5,), -7, dtype=dtype, device=DEV)
    return store[:n * k].view(n, k), store[n * k:]


def forward(z, token, k, T=1.0, view=None):
    """Calls the operator on z (CPU) and checks all it writes; returns the device's lse and entropy."""
    n, V = z.shape
    view = z.to(DEV) if view is None else view
    m = 0 if token is None else token.shape[1]
    logp, rank, ent, lse, idx, val = (padded(n, w, t) for w, t in ((m, F32), (1, torch.int32), (1, F32), (1, F32), (k, torch.int32), (k, F32)))
    gk.gk_vocab_logprob(view, None if token is None else token.to(DEV), logp_out=None if m == 0 else logp[0], rank_out=rank[0][:, 0],
                        entropy_out=ent[0][:, 0], lse_out=lse[0][:, 0], idx_out=idx[0] if k else None, val_out=val[0] if k else None,
                        temperature=T)
    torch.cuda.synchronize()
    for out, behind in (logp, rank, ent, lse, idx, val):
        assert bool((behind == -7).all())
    ref = reference(z, token, T, k)
    tol = bounds(z, ref, T)
    assert close(lse[0][:, 0], ref["lse"], tol["lse"])
    assert close(ent[0][:, 0], ref["entropy"], tol["entropy"])
    assert torch.equal(rank[0][:, 0].cpu().long(), ref["rank"])
    if m:
        assert close(logp[0], ref["logp"], logp_tol(ref["logp"]))
    if k:
        assert torch.equal(idx[0].cpu().long(), ref["idx"])
        assert close(val[0], ref["val"], logp_tol(ref["val"]))
    return lse[0][:, 0].contiguous(), ent[0][:, 0].contiguous()


def backward(z, token, T, lse, entropy, a, b, c, view=None, out=None):
    n, V = z.shape
    view = z.to(DEV) if view is None else view
    out = torch.empty(n, V, dtype=z.dtype, device=DEV) if out is None else out
    put = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    gk.gk_vocab_logprob_grad(view, put(token), lse, out, logp_grad=put(a), entropy=entropy if b is not None else None,
                             entropy_grad=put(b), lse_grad=put(c), temperature=T)
    want, tol = grad_reference(z, token, T, lse.cpu(), entropy.cpu(), a, b, c)
    u = torch.finfo(z.dtype).eps / 2
    tiny = {F32: 2.0 ** -126, BF16: 2.0 ** -126, F16: 2.0 ** -25}[z.dtype]      # powers below fp32's normal range are zero
    assert close(out, want, tol + u * (want.abs() + tol) + tiny)
    return out


def tokens_for(n, V, m, gen):
    t = torch.randint(0, V, (n, m), generator=gen)
    if n > 2:
        t[1] = -100                       # left out
        t[2, 0] = V + 3                   # out of range
        if m > 1:
            t[2, 1] = V - 1
    if m > 2:
        t[0, 2] = t[0, 0]                 # the same twice
    return t


SIZES = [(1, 1, 1, 1), (3, 2, 1, 2), (1, 7, 0, 3), (5, 33, 2, 20), (4, 1000, 1, 1), (3, 1025, 3, 128), (2, 4097, 1, 64), (7, 10000, 5, 0),
         (3, 32000, 1, 100), (4, 50001, 1, 20), (2, 200003, 128, 128), (300, 515, 1, 9), (700, 3001, 1, 5)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,m,k", SIZES)
def test_random_rows_forward_and_backward(n, V, m, k, dtype):
    gen = torch.Generator().manual_seed(n + V + k)
    z = (torch.randn(n, V, generator=gen) * 3).to(dtype)
    T = 1.0 if (n + k) % 2 else 0.7
    T = float(torch.tensor(T, dtype=F32))
    token = tokens_for(n, V, m, gen) if m else None
    lse, entropy = forward(z, token, k, T)
    a = torch.randn(n, m, generator=gen) if m else None
    b, c = torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    backward(z, token, T, lse, entropy, a, b, c)
    if m:
        backward(z, token, T, lse, entropy, a, None, None)
    backward(z, token, T, lse, entropy, None, b, None)


@pytest.mark.parametrize("dtype", TYPES)
def test_confident_rows(dtype):
    """Nearly all the mass on one token: the entropy and the log probability are small numbers of their own."""
    gen = torch.Generator().manual_seed(2)
    z = torch.randn(6, 5000, generator=gen)
    z[torch.arange(6), torch.arange(6) * 800 + 3] = torch.tensor([12.0, 16.0, 20.0, 30.0, 60.0, 200.0])
    token = (torch.arange(6) * 800 + 3)[:, None]
    lse, entropy = forward(z.to(dtype), token, 4)
    backward(z.to(dtype), token, 1.0, lse, entropy, torch.ones(6, 1), torch.ones(6), None)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_rows_infinities_and_nan(dtype):
    gen = torch.Generator().manual_seed(4)
    for V in (60, 3000, 30000):
        z = (torch.randn(10, V, generator=gen) * 2).to(dtype)
        z[0] = -math.inf                                   # nothing left
        z[1, 5:] = -math.inf                               # fewer than k left
        z[2, torch.rand(V, generator=gen) < 0.9] = -math.inf
        z[3] = torch.finfo(dtype).min                      # the type's lowest value
        z[4, 11] = math.inf
        z[5, 13] = math.nan
        z[6, ::2] = 0.0
        z[6, 1::2] = -0.0
        z[7, :40] = torch.finfo(dtype).max
        z[8, 7:] = torch.finfo(dtype).min
        z[9, 3], z[9, 40] = math.inf, math.nan
        token = torch.randint(0, V, (10, 3), generator=gen)
        token[4, 1], token[5, 1], token[2, 2] = 11, 13, 0
        lse, entropy = forward(z, token, 33)
        rows = [0, 1, 2, 3, 6, 7, 8]                       # the gradients of the others are what the formula gives
        backward(z[rows], token[rows], 1.0, lse[rows], entropy[rows], torch.randn(7, 3, generator=gen), torch.randn(7, generator=gen),
                 torch.randn(7, generator=gen))


def test_a_row_of_infinities_or_nan_spoils_no_other():
    z = torch.randn(4, 300)
    z[1, 5], z[2, 7] = math.nan, math.inf
    token = torch.tensor([[1], [2], [3], [4]])
    lse, entropy = forward(z, token, 3)
    out = torch.empty(4, 300, device=DEV)
    gk.gk_vocab_logprob_grad(z.to(DEV), token.to(DEV), lse, out, logp_grad=torch.ones(4, 1, device=DEV), entropy=entropy,
                             entropy_grad=torch.ones(4, device=DEV))
    bad = torch.isnan(out).any(1).cpu()
    assert bad.tolist() == [False, True, True, False]
    # rows that are left out are zero whatever they hold
    token[1:3] = -1
    forward(z, token, 3)
    gk.gk_vocab_logprob_grad(z.to(DEV), token.to(DEV), lse, out, logp_grad=torch.full((4, 1), math.nan, device=DEV))
    assert bool((out[1:3] == 0).all()) and bool(torch.isnan(out[0]).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_go_to_the_lower_index(dtype):
    gen = torch.Generator().manual_seed(3)
    for levels in (1, 2, 5):
        for V, k in ((700, 50), (20000, 128), (40000, 3)):
            z = torch.randint(0, levels, (3, V), generator=gen).to(dtype)
            token = torch.randint(0, V, (3, 1), generator=gen)
            forward(z, token, k)
            forward(-z * 0.5, token, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("order", ["ascending", "descending", "one_block", "few_above"])
def test_rows_in_an_order(order, dtype):
    """The largest last, first, within a short stretch; fewer above the rest than are asked for."""
    V = 30011
    z = torch.linspace(-9, 9, V).repeat(2, 1)
    if order == "descending":
        z = z.flip(1).contiguous()
    if order == "one_block":
        z = torch.zeros(2, V)
        z[:, 17000:17800] = torch.randn(2, 800, generator=torch.Generator().manual_seed(1)).abs() + 1
    if order == "few_above":
        z = torch.full((2, V), torch.finfo(dtype).min)
        z[:, 25000:25007] = 1.0
    forward(z.to(dtype), torch.tensor([[17], [V - 1]]), 100)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift,out_pad,out_shift", [(0, 1, 0, 1), (3, 0, 3, 0), (8, 5, 0, 0), (1, 0, 2, 3)])
def test_row_strides_and_unaligned_rows(pad, shift, out_pad, out_shift, dtype):
    gen = torch.Generator().manual_seed(6)
    n, V = 5, 5003
    z = (torch.randn(n, V, generator=gen) * 2).to(dtype)
    store = torch.full((n * (V + pad) + shift,), 1e4, dtype=dtype, device=DEV)
    view = store[shift:].view(n, V + pad)[:, :V]
    view.copy_(z)
    token = tokens_for(n, V, 3, gen)
    lse, entropy = forward(z, token, 40, view=view)
    keep = torch.full((n * (V + out_pad) + out_shift,), 7.0, dtype=dtype, device=DEV)
    out = keep[out_shift:].view(n, V + out_pad)[:, :V]
    args = torch.randn(n, 3, generator=gen), torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    backward(z, token, 1.0, lse, entropy, *args, view=view, out=out)
    assert bool((keep[:out_shift] == 7).all()) and bool((keep[out_shift:].view(n, -1)[:, V:] == 7).all())
    # in place
    apart = out.clone()
    backward(z, token, 1.0, lse, entropy, *args, view=view, out=view)
    assert torch.equal(view, apart)
    assert bool((store[:shift] == 1e4).all()) and bool((store[shift:].view(n, -1)[:, V:] == 1e4).all())


@pytest.mark.parametrize("T", [1e-3, 0.37, 40.0, 1e30])
def test_temperatures(T):
    T = float(torch.tensor(T, dtype=F32))
    gen = torch.Generator().manual_seed(8)
    z = torch.randn(4, 3000, generator=gen)
    token = torch.randint(0, 3000, (4, 1), generator=gen)
    lse, entropy = forward(z, token, 5, T)
    backward(z, token, T, lse, entropy, torch.randn(4, 1, generator=gen), torch.randn(4, generator=gen), None)


def test_the_gradient_against_differences():
    """Of a sum of all outputs with random weights: (f(z + e) - f(z - e)) / 2e in 64 bits, whose own error is e^2 f'''."""
    gen = torch.Generator().manual_seed(9)
    n, V, T, e = 3, 41, 0.8, 1e-4
    z = torch.randn(n, V, generator=gen)
    token = torch.tensor([[3, 7], [40, 40], [0, -1]])
    a, b, c = torch.randn(n, 2, generator=gen), torch.randn(n, generator=gen), torch.randn(n, generator=gen)

    def f(x):
        y = x / float(torch.tensor(T, dtype=F32))
        logp = torch.log_softmax(y, 1)
        ok = token >= 0
        return ((logp.gather(1, token.clamp(min=0)) * a.double())[ok].sum() + (b.double() * -(logp.exp() * logp).sum(1)).sum()
                + (c.double() * torch.logsumexp(y, 1)).sum())

    want = torch.empty(n, V, dtype=torch.float64)
    for i in range(n):
        for v in range(V):
            step = torch.zeros(n, V, dtype=torch.float64)
            step[i, v] = e
            want[i, v] = (f(z.double() + step) - f(z.double() - step)) / (2 * e)
    lse, entropy = forward(z, token, 0, float(torch.tensor(T, dtype=F32)))
    out = torch.empty(n, V, device=DEV)
    gk.gk_vocab_logprob_grad(z.to(DEV), token.to(DEV), lse, out, logp_grad=a.to(DEV), entropy=entropy, entropy_grad=b.to(DEV),
                             lse_grad=c.to(DEV), temperature=T)
    # third derivatives are below 40 here (1 / T^3 = 2, sums of |a|, |b| log p and |c| below 20); fp32 below 1e-5 of it
    assert float((out.cpu().double() - want).abs().max()) <= 40 * e * e + 1e-4


def test_offsets_past_32_bits():
    n, V, k = 17000, 130001, 5          # 2.2e9 logits
    gen = torch.Generator(device=DEV).manual_seed(7)
    z = torch.empty(n, V, dtype=BF16, device=DEV)
    for r in range(0, n, 1000):
        z[r:r + 1000] = torch.randn(1000, V, generator=gen, device=DEV).bfloat16()
    token = torch.randint(0, V, (n, 1), generator=gen, device=DEV)
    logp, lse, ent = (torch.empty(n, device=DEV) for _ in range(3))
    idx, val = torch.empty(n, k, dtype=torch.int32, device=DEV), torch.empty(n, k, device=DEV)
    gk.gk_vocab_logprob(z, token, logp_out=logp, entropy_out=ent, lse_out=lse, idx_out=idx, val_out=val)
    a = torch.ones(n, 1, device=DEV)
    some = [0, 1, 8000, n - 2, n - 1]
    rows = z[some].cpu()
    gk.gk_vocab_logprob_grad(z, token, lse, z, logp_grad=a, entropy=ent, entropy_grad=a[:, 0].contiguous())
    ref = reference(rows, token[some].cpu(), 1.0, k)
    assert torch.equal(idx[some].cpu().long(), ref["idx"])
    assert close(logp[some][:, None], ref["logp"], logp_tol(ref["logp"])) and close(lse[some], ref["lse"], bounds(rows, ref, 1.0)["lse"])
    want, tol = grad_reference(rows, token[some].cpu(), 1.0, lse[some].cpu(), ent[some].cpu(), torch.ones(5, 1), torch.ones(5), None)
    assert close(z[some], want, tol + 2.0 ** -8 * (want.abs() + tol) + 2.0 ** -126)


def test_outputs_that_are_not_wanted_and_no_rows():
    z = torch.randn(3, 500, device=DEV)
    token = torch.tensor([1, 2, 3], device=DEV)
    logp = torch.empty(3, device=DEV)
    gk.gk_vocab_logprob(z, token, logp_out=logp)
    want = torch.log_softmax(z.double(), 1).gather(1, token[:, None])[:, 0]
    assert close(logp, want.cpu(), logp_tol(want.cpu()))
    gk.gk_vocab_logprob(z, None)
    gk.gk_vocab_logprob(z[:0], token[:0], logp_out=logp[:0])
    gk.gk_vocab_logprob_grad(z[:0], token[:0], logp[:0], z[:0], logp_grad=logp[:0])


def test_replays_and_other_streams():
    n, V = 37, 8000
    gen = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn(n, V, generator=gen, device=DEV).bfloat16()
    token = torch.randint(0, V, (n, 1), generator=gen, device=DEV)
    bufs = lambda: [torch.empty(n, device=DEV) for _ in range(3)] + [torch.empty(n, 7, dtype=torch.int32, device=DEV), torch.empty(n, 7, device=DEV), torch.empty_like(z)]  # noqa: E731

    def call(out):
        gk.gk_vocab_logprob(z, token, logp_out=out[0], entropy_out=out[1], lse_out=out[2], idx_out=out[3], val_out=out[4])
        gk.gk_vocab_logprob_grad(z, token, out[2], out[5], logp_grad=torch.ones_like(out[0]), entropy=out[1], entropy_grad=out[0])

    replayed, stream = bufs(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call(replayed)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(replayed)
    for seed in (3, 4):
        z.copy_(torch.randn(n, V, generator=gen, device=DEV) * seed)
        eager = bufs()
        call(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, replayed))


def test_refusals():
    z = torch.zeros(2, 50, device=DEV)
    token = torch.zeros(2, 1, dtype=torch.int64, device=DEV)
    f = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731
    i = lambda *s: torch.empty(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    for args, kw in (((z.double(), token), {}), ((z.cpu(), token), {}), ((z[0], token), {}), ((z.t(), token), {}), ((z, token.int()), {}),
                     ((z, token[:1]), {}), ((z, token.cpu()), {}), ((z, token), {"logp_out": f(3)}), ((z, token), {"rank_out": f(2)}),
                     ((z, token), {"idx_out": i(2, 4)}), ((z, token), {"idx_out": i(2, 51), "val_out": f(2, 51)}),
                     ((torch.zeros(2, 500, device=DEV), token), {"idx_out": i(2, 129), "val_out": f(2, 129)}),
                     ((z, token), {"idx_out": i(2, 4), "val_out": f(2, 5)}), ((z, token), {"temperature": 0.0}), ((z, token), {"temperature": math.nan}),
                     ((z, torch.zeros(2, 129, dtype=torch.int64, device=DEV)), {}), ((z, None), {"logp_out": f(2)})):
        with pytest.raises(gk.GkError):
            gk.gk_vocab_logprob(*args, **kw)
    lse = f(2)
    for args, kw in (((z, token, lse, z.bfloat16()), {}), ((z, token, lse, f(2, 49)), {}), ((z, token, None, f(2, 50)), {}),
                     ((z, token, f(3), f(2, 50)), {}), ((z, token, lse, f(2, 50)), {"logp_grad": f(2, 2)}),
                     ((z, token, lse, f(2, 50)), {"entropy_grad": f(2)}), ((z, None, lse, f(2, 50)), {"logp_grad": f(2, 0)}),
                     ((z, token, lse, f(2, 50)), {"temperature": -1.0}), ((z[:, :40], token, lse, z[:, 10:]), {})):
        with pytest.raises(gk.GkError):
            gk.gk_vocab_logprob_grad(*args, **kw)
