"""Where the vocabulary head's operators can go wrong beyond sizes."""
import math

import pytest
import torch

from paper_1911_08772_b200 import binding as gk
from test_gpu_vocab_head import DEV, TYPES, Out, _library, check, distill, hard_loss, make  # noqa: F401  (_library: a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture
def budget():
    yield gk.gk_vocab_set_budget
    gk.gk_vocab_set_budget(2 << 30)


# --- one part of the vocabulary after another -------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dw", [True, False])
@pytest.mark.parametrize("V,columns", [(2100, 2048), (4100, 4096), (4200, 4096)])
def test_a_last_piece_of_fewer_blocks_than_dh_has_parts(V, columns, dw, dtype, budget):
    """dh's sum over the vocabulary is split into parts by the full piece (here at least four); the last piece has
    one or two blocks of 64 columns."""
    budget(2 * 256 * columns)
    hard_loss(200, 136, V, dtype, seed=60, left_out=0.1, dw=dw)
    distill(200, 136, V, 9, dtype, seed=61, dw=dw)


@pytest.mark.parametrize("dtype", TYPES)
def test_columns_past_the_end_of_logits_far_below_zero(dtype, budget):
    """With all logits near -200 the columns past the vocabulary's end, whose sums are 0, are far above the rest:
    nothing of them may reach a gradient, in one piece or in the last of several, nor of what a call before, of a
    vocabulary that ends on 16 bytes, left there."""
    n, D = 200, 72
    for V, columns in ((1301, 4096), (1301, 512), (1283, 256)):
        budget(2 * 256 * columns)
        _, _, _, hd, wd = make(n, D, (V + 7) // 8 * 8, dtype, 62)
        last = Out(n, D, (V + 7) // 8 * 8, dtype)
        gk.gk_vocab_loss(hd, wd, torch.zeros(n, dtype=torch.int64, device=DEV), last.loss[:n], last.lse[:n],
                         row_grad=torch.full((n,), math.nan, device=DEV), dh=last.dh, dw=last.dw)
        assert bool(torch.isnan(last.dw).all())
        gen, h, w, hd, wd = make(n, D, V, dtype, 62)
        h[:, 0] = 1.0
        w[:, 0] = -200.0
        hd.copy_(h)
        wd.copy_(w)
        target = torch.randint(0, V, (n,), generator=gen)
        g = torch.randn(n, generator=gen)
        out = Out(n, D, V, dtype)
        gk.gk_vocab_loss(hd, wd, target.to(DEV), out.loss[:n], out.lse[:n], row_grad=g.to(DEV), dh=out.dh, dw=out.dw)
        one = torch.ones(n, 1, dtype=torch.float64)
        check(out, h, w, target[:, None], one, torch.zeros_like(one), 1.0, g.double(), torch.ones(n, dtype=torch.bool), dtype)


# --- lanes of a reading warp that find something and lanes that do not ------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [769, 1600, 2400])
def test_few_rows_of_a_warp_have_pairs_in_a_tile(D, dtype):
    """Over 768 the logits are summed in chunks, and a row's first pair is looked up between two of them, by the
    lanes whose rows have one there."""
    hard_loss(70, D, 900, dtype, seed=67, left_out=0.2)
    distill(70, D, 900, 3, dtype, seed=68)
    distill(33, D, 300, 40, dtype, seed=69, holes=0.7)
    distill(70, D, 900, 3, dtype, seed=70, dh=False, dw=False)


# --- rows that are not finite -----------------------------------------------------------------------------


@pytest.mark.parametrize("V", [300, 20000])
@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("n", [1, 9, 40])
def test_a_row_of_nan_that_counts_has_a_log_sum_exp_of_nan(n, grad, V):
    D = 64
    gen, h, w, hd, wd = make(n, D, V, torch.bfloat16, 63)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)
    g = torch.ones(n, device=DEV)
    bad = n // 2
    base, out = (Out(n, D, V, torch.bfloat16, dh=grad, dw=False) for _ in range(2))
    gk.gk_vocab_loss(hd, wd, target, base.loss[:n], base.lse[:n], dh=base.dh, row_grad=g)
    hd[bad] = math.nan
    gk.gk_vocab_loss(hd, wd, target, out.loss[:n], out.lse[:n], dh=out.dh, row_grad=g)
    rest = torch.arange(n, device=DEV) != bad
    assert bool(torch.isnan(out.loss[bad])) and bool(torch.isnan(out.lse[bad]))
    assert torch.equal(out.loss[:n][rest], base.loss[:n][rest]) and torch.equal(out.lse[:n][rest], base.lse[:n][rest])
    if grad:
        assert torch.equal(out.dh[rest], base.dh[rest]) and bool(torch.isnan(out.dh[bad]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [300, 1100])
@pytest.mark.parametrize("size", [1e-6, 128.0])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_a_row_gradient_that_is_not_finite_reaches_its_own_row_of_dh_only(value, size, n, dtype):
    """The rows share one scale, which the others' gradients set: their rows are those of the call with a zero in
    the bad row's place, bit by bit."""
    D, V, K, bad = 72, 500, 5, 17
    gen, h, w, hd, wd = make(n, D, V, dtype, 64)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)
    idx = torch.stack([torch.randperm(V, generator=gen)[:K].sort().values for _ in range(n)]).to(torch.int32).to(DEV)
    val = torch.randn(n, K, generator=gen).to(DEV)
    g = (torch.randn(n, generator=gen) * size).to(DEV)
    rest = torch.arange(n, device=DEV) != bad
    for soft in (False, True):
        dhs = []
        for x in (0.0, value) + ((3e38,) if soft else ()):       # at T = 0.5 the last is infinite too
            g[bad] = x
            out = Out(n, D, V, dtype)
            if soft:
                gk.gk_vocab_distill(hd, wd, idx, val, out.loss[:n], out.lse[:n], temperature=0.5, row_grad=g, dh=out.dh, dw=out.dw)
            else:
                gk.gk_vocab_loss(hd, wd, target, out.loss[:n], out.lse[:n], row_grad=g, dh=out.dh, dw=out.dw)
            dhs.append(out.dh[rest])
        assert bool(torch.isfinite(dhs[0]).all()) and bool((dhs[0] != 0).any())
        assert all(torch.equal(dhs[0], x) for x in dhs[1:])


def test_a_teacher_mass_that_is_not_finite_reaches_its_own_row_of_dh_only():
    n, D, V, K, bad = 300, 72, 500, 5, 17
    gen, h, w, hd, wd = make(n, D, V, torch.float16, 65)
    idx = torch.stack([torch.randperm(V, generator=gen)[:K].sort().values for _ in range(n)]).to(torch.int32).to(DEV)
    val = torch.randn(n, K, generator=gen).to(DEV)
    g = torch.full((n,), 128.0, device=DEV)
    lse = torch.logsumexp(val, 1)
    rest = torch.arange(n, device=DEV) != bad
    dhs = []
    for x in (float(lse[bad]), -math.inf, math.nan):
        lse[bad] = x
        out = Out(n, D, V, torch.float16)
        gk.gk_vocab_distill(hd, wd, idx, val, out.loss[:n], out.lse[:n], t_lse=lse, row_grad=g, dh=out.dh, dw=out.dw)
        dhs.append(out.dh[rest])
    assert bool(torch.isfinite(dhs[0]).all())
    assert torch.equal(dhs[0], dhs[1]) and torch.equal(dhs[0], dhs[2])


# --- the workspace ----------------------------------------------------------------------------------------


@pytest.mark.parametrize("n,fewer,D,V", [(700, [700, 449, 200, 65, 1], 512, 9000), (2048, [1537, 1025, 300], 2048, 8000)])
def test_a_workspace_reserved_for_more_rows_can_be_captured_with_fewer(n, fewer, D, V):
    """A call that had to replace the workspace could not be captured: neither the wait nor the allocation may be."""
    gen, h, w, hd, wd = make(n, D, V, torch.bfloat16, 71)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        gk.gk_vocab_reserve(n, D, V)
        for m in fewer:
            for dw in (False, True):
                eager, out = (Out(m, D, V, torch.bfloat16, dw=dw) for _ in range(2))
                graph = torch.cuda.CUDAGraph()
                stream.synchronize()
                with torch.cuda.graph(graph, stream=stream):
                    gk.gk_vocab_loss(hd[:m], wd, target[:m], out.loss[:m], out.lse[:m], dh=out.dh, dw=out.dw)
                graph.replay()
                gk.gk_vocab_loss(hd[:m], wd, target[:m], eager.loss[:m], eager.lse[:m], dh=eager.dh, dw=eager.dw)
                stream.synchronize()
                assert torch.equal(out.loss, eager.loss) and torch.equal(out.dh, eager.dh)
                assert not dw or torch.equal(out.dw, eager.dw)


def test_a_first_call_within_a_capture_that_may_allocate():
    """In a capture in relaxed mode the stream's first call makes its workspace; replays are the eager call's."""
    n, D, V = 50, 72, 500
    gen, h, w, hd, wd = make(n, D, V, torch.bfloat16, 73)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)
    eager, out = Out(n, D, V, torch.bfloat16), Out(n, D, V, torch.bfloat16)
    gk.gk_vocab_loss(hd, wd, target, eager.loss[:n], eager.lse[:n], dh=eager.dh, dw=eager.dw)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream(priority=-1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream, capture_error_mode="relaxed"):
        gk.gk_vocab_loss(hd, wd, target, out.loss[:n], out.lse[:n], dh=out.dh, dw=out.dw)
    for _ in range(2):
        out.dh.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.loss, eager.loss) and torch.equal(out.dh, eager.dh) and torch.equal(out.dw, eager.dw)


# --- calls without rows -----------------------------------------------------------------------------------


def test_a_call_without_rows_is_the_last_call():
    w = torch.ones(30, 16, dtype=torch.bfloat16, device=DEV)
    none = (torch.empty(0, 16, dtype=torch.bfloat16, device=DEV), w, torch.empty(0, dtype=torch.int64, device=DEV))
    e, f = torch.empty(0, device=DEV), torch.empty(3, device=DEV)
    stream = torch.cuda.Stream(priority=-1)       # (no other test's: torch deals streams out in turn)
    with torch.cuda.stream(stream):
        with pytest.raises(gk.GkError):
            gk.gk_vocab_last_info()                       # no call yet
        gk.gk_vocab_loss(*none, e, e, dw=torch.ones_like(w))
        assert gk.gk_vocab_last_info() == (0, 0)
        gk.gk_vocab_reserve(3, 16, 30)
        assert gk.gk_vocab_last_info() == (0, 0)
        gk.gk_vocab_loss(w[:3], w, torch.zeros(3, dtype=torch.int64, device=DEV), f, f.clone())
        assert gk.gk_vocab_last_info() == (0, 3)
        gk.gk_vocab_loss(*none, e, e, dw=torch.ones_like(w))
        assert gk.gk_vocab_last_info() == (0, 0)
        gk.gk_vocab_loss(w[:3], w, torch.zeros(3, dtype=torch.int64, device=DEV), f, f.clone())
        assert gk.gk_vocab_last_info() == (0, 3)
        gk.gk_vocab_reserve(3000, 16, 30)                 # a larger block: the last call stays the last
        assert gk.gk_vocab_last_info() == (0, 3)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            gk.gk_vocab_loss(w[:5], w, torch.zeros(5, dtype=torch.int64, device=DEV), torch.empty(5, device=DEV), torch.empty(5, device=DEV))
        gk.gk_vocab_loss(*none, e, e, dw=torch.ones_like(w))
        assert gk.gk_vocab_last_info() == (0, 0)
        graph.replay()
        assert gk.gk_vocab_last_info() == (0, 5)
    other = torch.cuda.Stream(priority=-1)
    with torch.cuda.stream(other):
        gk.gk_vocab_reserve(3, 16, 30)
        with pytest.raises(gk.GkError):
            gk.gk_vocab_last_info()


# --- numbers ----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,V,K", [(1, 16, 5, 1), (3, 65, 300, 300), (130, 72, 515, 7), (1100, 64, 3000, 40), (64, 136, 20000, 100)])
def test_distillation_without_gradients(n, D, V, K, dtype):
    distill(n, D, V, K, dtype, seed=n + K, T=1.0 if n % 2 else 2.0, mass=n % 3 == 0, dh=False, dw=False)
    distill(n, D, V, K, dtype, seed=n + K + 1, T=1.5, mass=n % 3 != 0, holes=0.4, dh=False, dw=False)


def off_by(got, want, dtype):
    """How far `got` is from `want` (64 bits) in units of what want rounded to the type is off by, as norms."""
    want = want.cpu()
    return float((got.cpu().double() - want).norm() / (want.to(dtype).double() - want).norm())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("soft", [False, True])
@pytest.mark.parametrize("n,D,V,columns", [(1000, 200, 3000, 0), (600, 256, 20000, 0), (600, 256, 20000, 4096)])
def test_gradients_are_rounded_twice_and_no_more(n, D, V, columns, soft, dtype, budget):
    """As norms over many rows the errors of independent roundings add as squares: a logit gradient's (1), what is
    kept of a logit (0.48 of one in bf16: 3.9e-4 against 8.1e-4 root mean square, 0.25 in fp16) and the result's
    own (1): at most sqrt(2.23) = 1.49 times the last alone.  One rounding more would be 1.79 (1.75).  (The bounds
    element by element in vocab_util.py leave room for it.)"""
    if columns:
        budget(2 * 768 * columns)
    gen, h, w, hd, wd = make(n, D, V, dtype, 66)
    K = 30 if soft else 1
    idx = torch.stack([torch.randperm(V, generator=gen)[:K].sort().values for _ in range(n)])
    t = torch.randn(n, K, generator=gen) * 2
    q = torch.softmax(t.double(), 1)
    out = Out(n, D, V, dtype)
    g = torch.rand(n, generator=gen) + 0.5
    if soft:
        gk.gk_vocab_distill(hd, wd, idx.to(torch.int32).to(DEV), t.to(DEV), out.loss[:n], out.lse[:n], row_grad=g.to(DEV), dh=out.dh, dw=out.dw)
    else:
        gk.gk_vocab_loss(hd, wd, idx[:, 0].to(DEV), out.loss[:n], out.lse[:n], row_grad=g.to(DEV), dh=out.dh, dw=out.dw)
    hx, wx, gx, qx = (x.double().to(DEV) for x in (h, w, g, q))
    dz = torch.softmax(hx @ wx.t(), 1)
    dz.scatter_add_(1, idx.to(DEV), -qx)
    dz *= gx[:, None]
    assert off_by(out.dh, dz @ wx, dtype) <= 1.6
    assert off_by(out.dw, dz.t() @ hx, dtype) <= 1.6


# --- calls one after another ------------------------------------------------------------------------------


@pytest.mark.parametrize("n,D,V", [(300, 200, 1501), (1100, 72, 3000), (64, 136, 20000)])
def test_calls_that_read_what_the_call_before_wrote(n, D, V):
    """The kernels of a call are set up while the one before them runs: without a wait between calls, over buffers
    that each call writes anew, the results are those of calls with a wait after each."""
    gen = torch.Generator(device=DEV).manual_seed(72)
    w = (torch.randn(V, D, generator=gen, device=DEV) / 4).bfloat16()
    hs = [torch.randn(n, D, generator=gen, device=DEV).bfloat16() for _ in range(6)]
    zs = [torch.randn(n, V, generator=gen, device=DEV) * 3 for _ in range(6)]
    K = 20

    def steps(wait):
        t_idx, t_val, t_lse = torch.empty(n, K, dtype=torch.int32, device=DEV), torch.empty(n, K, device=DEV), torch.empty(n, device=DEV)
        x = torch.empty(n, D, dtype=torch.bfloat16, device=DEV)
        loss, lse, dh, dw = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.zeros_like(x), torch.zeros_like(w)
        got = []
        for h, z in zip(hs, zs):
            x.copy_(h)
            for call in (lambda: gk.gk_vocab_topk(z, K, t_idx, t_val, lse_out=t_lse),
                         lambda: gk.gk_vocab_distill(x, w, t_idx, t_val, loss, lse, t_lse=t_lse, dh=dh, dw=dw),
                         lambda: gk.gk_vocab_loss(dh, dw, t_idx[:, 3].long(), loss, lse, dh=x),       # the gradients as inputs
                         lambda: gk.gk_vocab_loss(x, w, t_idx[:, 0].long(), loss, lse, dh=dh, dw=dw)):
                call()
                if wait:
                    torch.cuda.synchronize()
                got += [loss.clone(), lse.clone(), dh.clone(), x.clone(), dw.clone()]
        torch.cuda.synchronize()
        return got

    for a, b in zip(steps(True), steps(False)):
        assert torch.equal(a, b)
