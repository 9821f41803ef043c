"""The vocabulary head's losses (gk_vocab_loss, gk_vocab_distill) against the formulas in 64 bits:
sizes around the tiles' edges, rows left out, strides, pieces of the vocabulary, both types."""
import math

import pytest
import torch

from paper_1911_08772_b200 import binding as gk
from vocab_util import bounds, head_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield
    gk.gk_vocab_set_budget(2 << 30)


def rows_tensor(n, cols, dtype, pad=0, shift=0):
    """An (n, cols) view with row stride cols + pad that starts `shift` elements into its storage."""
    store = torch.full((n * (cols + pad) + shift + 8,), 7.0, dtype=dtype, device=DEV)
    return store, store[shift:shift + n * (cols + pad)].view(n, cols + pad)[:, :cols]


def make(n, D, V, dtype, seed, pad=0, shift=0):
    gen = torch.Generator().manual_seed(seed)
    h = torch.randn(n, D, generator=gen).to(dtype)
    w = (torch.randn(V, D, generator=gen) * (2.0 / math.sqrt(D))).to(dtype)
    _, hd = rows_tensor(n, D, dtype, pad, shift)
    _, wd = rows_tensor(V, D, dtype, pad, shift)
    hd.copy_(h)
    wd.copy_(w)
    return gen, h, w, hd, wd


class Out:
    """Result buffers filled with a mark, with guards after them."""

    def __init__(self, n, D, V, dtype, dh=True, dw=True, pad=0, shift=0):
        self.loss = torch.full((n + 4,), -77.0, device=DEV)
        self.lse = torch.full((n + 4,), -77.0, device=DEV)
        self.n, self.pad = n, pad
        self.dh_store, self.dh = rows_tensor(n, D, dtype, pad, shift) if dh else (None, None)
        self.dw_store, self.dw = rows_tensor(V, D, dtype, pad, shift) if dw else (None, None)

    def untouched(self):
        assert bool((self.loss[self.n:] == -77).all()) and bool((self.lse[self.n:] == -77).all())
        for store, t in ((self.dh_store, self.dh), (self.dw_store, self.dw)):
            if store is None:
                continue
            mask = torch.ones_like(store, dtype=torch.bool)
            off = t.storage_offset()
            rows, cols = t.shape
            if rows:
                mask[off:off + rows * (cols + self.pad)].view(rows, cols + self.pad)[:, :cols] = False
            assert bool((store[mask] == 7.0).all()), "a write outside the rows"


def check(out, h, w, idx, q, logq, T, g, on, dtype):
    """Rows not in `on` must be zero; the others within the bounds."""
    h0 = torch.where(on[:, None], h, torch.zeros_like(h))
    q = torch.where(on[:, None], q, torch.zeros_like(q))
    g = torch.where(on, g, torch.zeros_like(g))
    ref = head_reference(h0, w, idx, q, logq, T, g)
    tol = bounds(h0, w, ref, q, logq, T, dtype)
    n = h.shape[0]
    assert gk.gk_vocab_last_info() == (0, int(on.sum()))
    for name in ("loss", "lse"):
        got = getattr(out, name)[:n].cpu().double()
        want = torch.where(on, ref[name], torch.zeros_like(ref[name]))
        off = (got - want).abs().max().item()
        assert off <= tol[name], (name, off, tol[name])
        assert bool((got[~on] == 0).all())
    for name in ("dh", "dw"):
        t = getattr(out, name)
        if t is None:
            continue
        got = t.cpu().double()
        off = (got - ref[name]).abs() - tol[name]
        assert off.max().item() <= 0, (name, off.max().item(), (got - ref[name]).abs().max().item())
    if out.dh is not None:
        assert bool((out.dh.cpu()[~on] == 0).all())
    out.untouched()


def hard_loss(n, D, V, dtype, seed, left_out=0.0, pad=0, shift=0, dh=True, dw=True, mean=False, spoil=False):
    gen, h, w, hd, wd = make(n, D, V, dtype, seed, pad, shift)
    target = torch.randint(0, V, (n,), generator=gen)
    drop = torch.rand(n, generator=gen) < left_out
    target[drop] = torch.tensor([-100, -1, V, V + 5, 2 ** 40])[torch.randint(0, 5, (int(drop.sum()),), generator=gen)]
    on = ~drop
    if spoil:     # whatever a row that is left out holds
        bad = torch.tensor([math.nan, math.inf, -math.inf]).to(dtype)
        h[drop] = bad[torch.randint(0, 3, (int(drop.sum()), D), generator=gen)]
        hd.copy_(h)
    g = torch.randn(n, generator=gen) if not mean else torch.full((n,), 1.0 / max(1, int(on.sum())))
    out = Out(n, D, V, dtype, dh, dw, pad, shift)
    gk.gk_vocab_loss(hd, wd, target.to(DEV), out.loss[:n], out.lse[:n], row_grad=None if mean else g.to(DEV),
                     dh=out.dh, dw=out.dw)
    idx = target.clamp(0, V - 1)[:, None]
    check(out, h, w, idx, torch.ones(n, 1, dtype=torch.float64), torch.zeros(n, 1, dtype=torch.float64), 1.0, g.double(), on, dtype)


SIZES = [(1, 1, 1), (1, 8, 2), (2, 7, 3), (5, 64, 64), (33, 64, 255), (64, 72, 257), (127, 40, 700), (129, 200, 1000),
         (257, 129, 513), (300, 320, 2049), (513, 264, 300), (40, 1500, 777)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,V", SIZES)
def test_loss_and_gradients(n, D, V, dtype):
    hard_loss(n, D, V, dtype, seed=n + D + V)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("left_out", [0.3, 0.97, 1.0])
def test_rows_left_out_have_no_part_in_anything(left_out, dtype):
    hard_loss(300, 96, 600, dtype, seed=5, left_out=left_out, spoil=True)


@pytest.mark.parametrize("pad,shift", [(8, 0), (5, 0), (0, 1), (3, 3), (8, 8), (16, 4)])
def test_row_strides_and_unaligned_rows(pad, shift):
    hard_loss(70, 136, 401, torch.bfloat16, seed=6, pad=pad, shift=shift)
    hard_loss(70, 131, 401, torch.float16, seed=7, pad=pad, shift=shift)


@pytest.mark.parametrize("D,pad", [(131, 5), (136, 8), (1, 7), (60, 4)])
def test_what_lies_between_the_rows_does_not_matter(D, pad):
    n, V = 70, 401
    gen = torch.Generator().manual_seed(12)
    h, w = torch.randn(n, D, generator=gen).half().to(DEV), torch.randn(V, D, generator=gen).half().to(DEV)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)
    outs = []
    for fill in (0.0, math.nan):
        hp, wp = (torch.full((t.shape[0], D + pad), fill, dtype=torch.float16, device=DEV)[:, :D] for t in (h, w))
        hp.copy_(h)
        wp.copy_(w)
        out = Out(n, D, V, torch.float16)
        gk.gk_vocab_loss(hp, wp, target, out.loss[:n], out.lse[:n], dh=out.dh, dw=out.dw)
        outs.append(out)
    a, b = outs
    for x, y in ((a.loss, b.loss), (a.lse, b.lse), (a.dh, b.dh), (a.dw, b.dw)):
        assert torch.equal(x, y) and bool(torch.isfinite(x).all())


@pytest.mark.parametrize("dh,dw", [(True, False), (False, True), (False, False)])
def test_either_gradient_or_none(dh, dw):
    hard_loss(140, 128, 900, torch.bfloat16, seed=8, left_out=0.2, dh=dh, dw=dw)


def test_gradient_of_the_mean_over_the_rows_that_count():
    hard_loss(140, 128, 900, torch.bfloat16, seed=9, left_out=0.4, mean=True)
    hard_loss(140, 128, 900, torch.float16, seed=9, left_out=0.4, mean=True)


@pytest.mark.parametrize("budget", [0, 2 * 256 * 512, 2 * 256 * 768])
@pytest.mark.parametrize("dtype", TYPES)
def test_pieces_of_the_vocabulary(budget, dtype):
    gk.gk_vocab_set_budget(budget)
    try:
        hard_loss(200, 136, 1300, dtype, seed=10, left_out=0.1)
        distill(200, 136, 1300, 9, dtype, seed=11)
    finally:
        gk.gk_vocab_set_budget(2 << 30)


def distill(n, D, V, K, dtype, seed, T=1.0, mass=True, holes=0.0, repeats=False, dh=True, dw=True, scale=1.0):
    gen, h, w, hd, wd = make(n, D, V, dtype, seed)
    if repeats:
        idx = torch.randint(0, V, (n, K), generator=gen)
    else:
        idx = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(n)])
        idx[::2] = idx[::2].sort(1).values          # some rows ascending, as gk_vocab_topk writes them
    t = (torch.randn(n, K, generator=gen) * 2 + 3).float()
    count = torch.ones(n, K, dtype=torch.bool)
    if holes:
        count = torch.rand(n, K, generator=gen) >= holes
        kind = torch.randint(0, 3, (n, K), generator=gen)
        idx = torch.where(~count & (kind == 0), torch.full_like(idx, -1), idx)
        idx = torch.where(~count & (kind == 1), torch.full_like(idx, V), idx)
        t = torch.where(~count & (kind == 2), torch.full_like(t, -math.inf), t)
    td = torch.where(count, t.double() / T, torch.full((n, K), -math.inf, dtype=torch.float64))
    on = count.any(1)
    L = torch.logsumexp(td, 1)
    t_lse = None
    if mass:
        t_lse = (torch.where(on, L, torch.zeros_like(L)) + 0.3 * torch.rand(n, generator=gen)).float()
        L = t_lse.double()
    logq = torch.where(count, td - L[:, None], torch.zeros_like(td))
    q = torch.where(count, torch.exp(logq), torch.zeros_like(td))
    g = torch.randn(n, generator=gen) * scale
    out = Out(n, D, V, dtype, dh, dw)
    gk.gk_vocab_distill(hd, wd, idx.to(torch.int32).to(DEV), t.to(DEV), out.loss[:n], out.lse[:n],
                        t_lse=None if t_lse is None else t_lse.to(DEV), temperature=T, row_grad=g.to(DEV), dh=out.dh, dw=out.dw)
    check(out, h, w, idx.clamp(0, V - 1), q, logq, T, g.double(), on, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,V,K", [(1, 16, 5, 1), (3, 65, 300, 300), (130, 72, 515, 7), (259, 200, 1025, 33), (64, 520, 2000, 100)])
@pytest.mark.parametrize("mass", [True, False])
def test_distill(n, D, V, K, mass, dtype):
    distill(n, D, V, K, dtype, seed=n + K, T=1.0 if n % 2 else 2.0, mass=mass)


@pytest.mark.parametrize("mass", [True, False])
def test_distill_pairs_left_out_and_given_twice(mass):
    distill(150, 96, 700, 12, torch.bfloat16, seed=20, T=1.5, mass=mass, holes=0.5)
    distill(150, 96, 700, 3, torch.float16, seed=21, T=1.5, mass=mass, holes=0.8)
    distill(150, 96, 20, 12, torch.bfloat16, seed=22, T=0.7, mass=mass, repeats=True)
    distill(40, 64, 30, 1024, torch.bfloat16, seed=23, T=3.0, mass=mass, repeats=True, holes=0.1)


LARGE = [(1100, 72, 8000), (4500, 40, 2000), (130, 264, 70001)]      # 2^23 logits and more


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,V", LARGE)
def test_large_calls(n, D, V, dtype):
    hard_loss(n, D, V, dtype, seed=50, left_out=0.15, spoil=True)


@pytest.mark.parametrize("mass", [True, False])
def test_large_distillation(mass):
    distill(1100, 72, 8000, 40, torch.bfloat16, seed=51, T=1.5, mass=mass)
    distill(1100, 72, 8000, 12, torch.bfloat16, seed=52, T=0.8, mass=mass, holes=0.5)
    distill(2200, 64, 4000, 5, torch.bfloat16, seed=53, mass=mass, holes=0.3, repeats=True)


@pytest.mark.parametrize("budget", [0, 2 * 1280 * 3000])
def test_large_calls_in_pieces(budget):
    gk.gk_vocab_set_budget(budget)
    try:
        hard_loss(1100, 72, 8000, torch.bfloat16, seed=54, left_out=0.1)
        distill(1100, 72, 8000, 9, torch.bfloat16, seed=55)
    finally:
        gk.gk_vocab_set_budget(2 << 30)


@pytest.mark.parametrize("budget", [2 << 30, 2 * 1280 * 3000])
@pytest.mark.parametrize("low", [-40.0, -300.0])
def test_classes_far_below_the_rest(low, budget):
    """Losses up to some hundreds: a reference at the class is then no use for the row's powers.  The
    last column has some rows' highest logit, where a piece of its own may find it."""
    n, D, V = 1100, 72, 8000
    gen, h, w, hd, wd = make(n, D, V, torch.bfloat16, 56)
    h[:, 0] = 1.0
    w[:, 0] = 0.0
    target = torch.randint(0, V - 1, (n,), generator=gen)
    target[::3] = 5
    w[5, 0] = low
    w[V - 1] = 0.0
    w[V - 1, 0] = -low / 4
    hd.copy_(h)
    wd.copy_(w)
    g = torch.randn(n, generator=gen)
    out = Out(n, D, V, torch.bfloat16)
    gk.gk_vocab_set_budget(budget)
    try:
        gk.gk_vocab_loss(hd, wd, target.to(DEV), out.loss[:n], out.lse[:n], row_grad=g.to(DEV), dh=out.dh, dw=out.dw)
    finally:
        gk.gk_vocab_set_budget(2 << 30)
    check(out, h, w, target[:, None], torch.ones(n, 1, dtype=torch.float64), torch.zeros(n, 1, dtype=torch.float64), 1.0,
          g.double(), torch.ones(n, dtype=torch.bool), torch.bfloat16)


@pytest.mark.parametrize("scale", [1e-6, 1e5])
def test_gradients_of_rows_of_any_size(scale):
    """Row gradients far from 1: the 16-bit logit gradients are scaled to their type's range."""
    distill(150, 96, 700, 12, torch.bfloat16, seed=24, scale=scale)
    if scale > 1:
        scale = 100.0       # fp16 results end at 65504
    distill(150, 96, 700, 12, torch.float16, seed=25, scale=scale)


def test_no_rows():
    w = torch.ones(30, 16, dtype=torch.bfloat16, device=DEV)
    h = torch.empty(0, 16, dtype=torch.bfloat16, device=DEV)
    dw = torch.ones_like(w)
    e = torch.empty(0, device=DEV)
    gk.gk_vocab_loss(h, w, torch.empty(0, dtype=torch.int64, device=DEV), e, e, dw=dw)
    assert bool((dw == 0).all())


def test_differences_of_the_loss():
    """The loss itself at h +- step along a direction, against dh; and w +- step against dw.  All
    values are multiples of 2^-8 below 4, so that the moved points are exact in fp16.  Central
    differences are off by step^2 / 6 of the third derivative, at most (max_v |dz_v / dstep|)^3."""
    gen = torch.Generator().manual_seed(31)
    n, D, V = 40, 64, 333
    h = (torch.randint(-256, 257, (n, D), generator=gen) / 256.0)
    w = (torch.randint(-64, 65, (V, D), generator=gen) / 256.0)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)
    step = 2.0 ** -6
    dirh = (torch.randint(0, 2, (n, D), generator=gen) * 2 - 1) * (torch.rand(n, D, generator=gen) < 0.1)
    dirw = (torch.randint(0, 2, (V, D), generator=gen) * 2 - 1) * (torch.rand(V, D, generator=gen) < 0.1)

    def losses(hh, ww, grads=None):
        loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        kw = {} if grads is None else {"dh": grads[0], "dw": grads[1], "row_grad": torch.ones(n, device=DEV)}
        gk.gk_vocab_loss(hh.half().to(DEV), ww.half().to(DEV), target, loss, lse, **kw)
        return loss.cpu().double()

    dh = torch.empty(n, D, dtype=torch.float16, device=DEV)
    dw = torch.empty(V, D, dtype=torch.float16, device=DEV)
    losses(h, w, (dh, dw))
    noise = 2 * (D * 2.0 ** -23 * 20 + 2.0 ** -20 * 12) / (2 * step)      # of a difference of two losses
    u = 2.0 ** -11
    # per row along dirh
    num = (losses(h + step * dirh, w) - losses(h - step * dirh, w)) / (2 * step)
    an = (dh.cpu().double() * dirh).sum(1)
    move = (dirh.double() @ w.double().t()).abs().max().item()
    tol = noise + step ** 2 / 6 * 8 * move ** 3 + 4 * u * (2 * w.abs().max().item() * dirh.abs().sum(1).max().item())
    assert (num - an).abs().max().item() <= tol
    # the sum of the losses along dirw
    num = float((losses(h, w + step * dirw) - losses(h, w - step * dirw)).sum()) / (2 * step)
    an = float((dw.cpu().double() * dirw).sum())
    move = (h.double() @ dirw.double().t()).abs().max().item()
    tol = n * (noise + step ** 2 / 6 * 8 * move ** 3) + 4 * u * float((dw.cpu().double().abs() * dirw.abs()).sum() + 2 * n * move)
    assert abs(num - an) <= tol


def test_confident_rows_and_equal_logits():
    """Rows whose class has nearly all the mass, and rows whose logits are all equal."""
    n, D, V = 6, 64, 500
    w = torch.zeros(V, D)
    w[:, 0] = 1.0
    w[7, 1] = 8.0
    h = torch.zeros(n, D)
    h[:, 0] = 3.0
    h[3:, 1] = 5.0
    target = torch.tensor([7, 0, 499, 7, 7, 1])
    for dtype in TYPES:
        out = Out(n, D, V, dtype)
        g = torch.ones(n)
        gk.gk_vocab_loss(h.to(dtype).to(DEV), w.to(dtype).to(DEV), target.to(DEV), out.loss[:n], out.lse[:n], row_grad=g.to(DEV),
                         dh=out.dh, dw=out.dw)
        check(out, h.to(dtype), w.to(dtype), target[:, None], torch.ones(n, 1, dtype=torch.float64),
              torch.zeros(n, 1, dtype=torch.float64), 1.0, g.double(), torch.ones(n, dtype=torch.bool), dtype)


def test_the_same_call_gives_the_same_bits_on_any_stream_and_in_a_graph():
    n, D, V = 300, 200, 1500
    gen, h, w, hd, wd = make(n, D, V, torch.bfloat16, 40)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)
    first = Out(n, D, V, torch.bfloat16)

    def call(o):
        gk.gk_vocab_loss(hd, wd, target, o.loss[:n], o.lse[:n], dh=o.dh, dw=o.dw)

    def same(o):
        return all(torch.equal(a, b) for a, b in ((o.loss, first.loss), (o.lse, first.lse), (o.dh, first.dh), (o.dw, first.dw)))

    call(first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    second, third = Out(n, D, V, torch.bfloat16), Out(n, D, V, torch.bfloat16)
    with torch.cuda.stream(side):
        gk.gk_vocab_reserve(n, D, V, grad=True)
        call(second)
        side.synchronize()
        assert same(second)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(third)
        for o in (third.loss, third.lse, third.dh, third.dw):
            o.fill_(5.0) if o is not third.loss and o is not third.lse else o[:n].fill_(5.0)
        graph.replay()
        graph.replay()
        side.synchronize()
    assert same(third)


@pytest.mark.parametrize("n,D,V,K", [(30, 64, 500, 1), (700, 1500, 10000, 1), (2100, 512, 9000, 40), (300, 136, 70001, 7)])
def test_a_reserved_workspace_is_enough(n, D, V, K):
    gen, h, w, hd, wd = make(n, D, V, torch.bfloat16, 42)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        gk.gk_vocab_reserve(n, D, V, K, grad=True)
        assert gk.gk_vocab_workspace_bytes(n, D, V, K) > 0
        t_idx = torch.randint(0, V, (n, K), generator=gen).to(torch.int32).to(DEV)
        t_val = torch.randn(n, K, generator=gen).to(DEV)
        outs = [Out(n, D, V, torch.bfloat16, dh, dw, shift=shift) for dh, dw in ((True, True), (True, False), (False, True), (False, False))
                for shift in (0, 1)]
        stream.synchronize()
        free = torch.cuda.mem_get_info()[0]
        for out in outs:
            gk.gk_vocab_distill(hd, wd, t_idx, t_val, out.loss[:n], out.lse[:n], dh=out.dh, dw=out.dw)
        stream.synchronize()
        assert torch.cuda.mem_get_info()[0] == free
        assert gk.gk_vocab_last_info() == (0, n)


def test_offsets_past_32_bits():
    """2.5e9 logits in one piece: its bytes and its elements pass 2^32 and 2^31.  Some rows of dh and of dw
    against 64 bits, taking every row's log-sum-exp from a sample of rows that is checked itself."""
    n, D, V = 20000, 64, 125000
    gen = torch.Generator(device=DEV).manual_seed(43)
    h = torch.randn(n, D, generator=gen, device=DEV).bfloat16()
    w = (torch.randn(V, D, generator=gen, device=DEV) / 4).bfloat16()
    target = torch.randint(0, V, (n,), generator=gen, device=DEV)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    g = torch.ones(n, device=DEV)
    gk.gk_vocab_set_budget(6 << 30)
    try:
        gk.gk_vocab_loss(h, w, target, loss, lse, row_grad=g, dh=dh, dw=dw)
        assert gk.gk_vocab_last_info() == (0, n)
    finally:
        gk.gk_vocab_set_budget(2 << 30)
    rows = torch.cat([torch.arange(40), torch.arange(9990, 10030), torch.arange(n - 40, n)]).to(DEV)
    hr, wd = h[rows], w
    ref = head_reference(hr, wd, target[rows][:, None], torch.ones(len(rows), 1, dtype=torch.float64, device=DEV),
                         torch.zeros(len(rows), 1, dtype=torch.float64, device=DEV), 1.0, torch.ones(len(rows), dtype=torch.float64, device=DEV))
    one = torch.ones(len(rows), 1, dtype=torch.float64, device=DEV)
    tol = bounds(hr, wd, ref, one, torch.zeros_like(one), 1.0, torch.bfloat16)
    assert (loss[rows].double() - ref["loss"]).abs().max().item() <= tol["loss"]
    assert (lse[rows].double() - ref["lse"]).abs().max().item() <= tol["lse"]
    assert bool(((dh[rows].double() - ref["dh"]).abs() <= tol["dh"]).all())
    # dw's rows need every row's probability of their word: from the log-sum-exps, whose bound is in lse_tol
    words = torch.cat([torch.arange(20), torch.arange(62000, 62020), torch.arange(V - 20, V)]).to(DEV)
    p = torch.exp(h.double() @ w[words].double().t() - lse.double()[:, None])
    hard = (target[:, None] == words[None, :]).double()
    dz, size = p - hard, p + hard
    u = 2.0 ** -8
    dz_tol = (2 * u * (1 + u) + 8 * tol["lse"]) * size
    want = dz.t() @ h.double()
    bound = (dz_tol + n * 2.0 ** -23 * (size + dz_tol)).t() @ h.double().abs()
    assert bool(((dw[words].double() - want).abs() <= bound + u * (want.abs() + bound)).all())


def test_a_logit_of_infinity_reaches_its_own_row_only():
    n, D, V = 9, 64, 300
    _, h, w, hd, wd = make(n, D, V, torch.bfloat16, 41)
    target = torch.arange(n, device=DEV) * 3
    base, out = Out(n, D, V, torch.bfloat16, dw=False), Out(n, D, V, torch.bfloat16, dw=False)
    gk.gk_vocab_loss(hd, wd, target, base.loss[:n], base.lse[:n], dh=base.dh, row_grad=torch.ones(n, device=DEV))
    hd[4] = math.inf
    gk.gk_vocab_loss(hd, wd, target, out.loss[:n], out.lse[:n], dh=out.dh, row_grad=torch.ones(n, device=DEV))
    rest = torch.arange(n, device=DEV) != 4
    assert not bool(torch.isfinite(out.loss[4]))
    assert torch.equal(out.loss[:n][rest], base.loss[:n][rest]) and torch.equal(out.dh[rest], base.dh[rest])


def test_refusals():
    h = torch.zeros(4, 16, dtype=torch.bfloat16, device=DEV)
    w = torch.zeros(9, 16, dtype=torch.bfloat16, device=DEV)
    t = torch.zeros(4, dtype=torch.int64, device=DEV)
    f = torch.zeros(4, device=DEV)
    ok = lambda **kw: gk.gk_vocab_loss(**{**dict(h=h, w=w, target=t, loss_out=f, lse_out=f.clone()), **kw})  # noqa: E731
    for kw in (dict(h=h.float(), w=w.float()), dict(w=w.half()), dict(h=h.cpu()), dict(w=w[:, :8]), dict(target=t.int()),
               dict(target=t[:3]), dict(h=h.t().contiguous().t()), dict(h=h[:1].expand(4, 16)), dict(dh=h), dict(dw=w),
               dict(dh=torch.zeros(4, 16, device=DEV)), dict(dh=torch.zeros(3, 16, dtype=torch.bfloat16, device=DEV)),
               dict(row_grad=f.double()), dict(loss_out=f[:2]), dict(h=h[0])):
        with pytest.raises(gk.GkError):
            ok(**kw)
    ti, tv = torch.zeros(4, 2, dtype=torch.int32, device=DEV), torch.zeros(4, 2, device=DEV)
    good = dict(h=h, w=w, t_idx=ti, t_val=tv, loss_out=f, lse_out=f.clone())
    for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf),
               dict(t_idx=ti.long()), dict(t_val=tv[:, :1]), dict(t_lse=f[:1]),
               dict(t_idx=torch.zeros(4, 1025, dtype=torch.int32, device=DEV), t_val=torch.zeros(4, 1025, device=DEV))):
        with pytest.raises(gk.GkError):
            gk.gk_vocab_distill(**{**good, **kw})
