"""gk_grad_norm and gk_grad_clip against the definitions in 64 bits."""
import math

import pytest
import torch

from grad_util import NORM_TOL, check_clipped, check_norms, norms64, tensors
from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
LISTS = {"one": [1], "lone_row": [7], "few": [5, 1, 4096, 63, 64, 129], "empty_ones": [0, 17, 0, 0, 5000, 0],
         "long": [1_000_003, 3, 777_777], "many": [1 + (i * 37) % 900 for i in range(300)],
         "thousand": [64] * 1000, "past_the_argument": [1 + (i * 13) % 77 for i in range(2501)]}


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


def norm_of(grads):
    norm, norms = torch.full((3,), -7.0, device=DEV), torch.full((len(grads) + 3,), -7.0, device=DEV)
    gk.gk_grad_norm(grads, norm[:1], norms_out=norms[:len(grads)])
    assert bool((norm[1:] == -7).all()) and bool((norms[len(grads):] == -7).all())
    return norm[:1], norms[:len(grads)]


@pytest.mark.parametrize("types", [[F32], [BF16], [F16], [F32, BF16, F16]], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("name", LISTS)
def test_norms(name, types):
    grads = tensors(LISTS[name], types, seed=len(name))
    norm, norms = norm_of(grads)
    check_norms(grads, norm, norms)
    alone = torch.empty(1, device=DEV)
    gk.gk_grad_norm(gk.GradList(grads), alone)
    assert torch.equal(alone, norm)


@pytest.mark.parametrize("shift", [1, 3, 5])
@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_norms_of_unaligned_tensors(t, shift):
    grads = tensors([1, 2, 9, 4097, 70001], [t], shift=shift)
    check_norms(grads, *norm_of(grads))


@pytest.mark.parametrize("t,scale", [(F32, 1e25), (F32, 1e-30), (F32, 3e37), (F32, 1e-42), (BF16, 1e25), (BF16, 1e-30), (F16, 3e3), (F16, 1e-7)])
def test_squares_beyond_the_range_of_fp32(t, scale):
    """A square that overflows, one that is lost, and both beside ordinary values."""
    grads = tensors([5001, 64, 20000], [t], scale=scale)
    want = norms64(grads)
    norm, norms = norm_of(grads)
    total = float(want.square().sum().sqrt())
    tiny = 2.0 ** -149      # the results' smallest step

    def near(got, want):      # the largest draws are infinities themselves, and a norm can be one in fp32
        beyond = want > torch.finfo(F32).max
        return bool((torch.where(beyond, torch.isinf(got), (got.double() - want).abs() <= NORM_TOL * want + tiny)).all())

    assert near(norm.cpu(), torch.tensor([total], dtype=torch.float64)) and near(norms.cpu(), want)
    if math.isinf(total):
        return
    check_norms(grads + tensors([999], [t], scale=1.0), *norm_of(grads + tensors([999], [t], scale=1.0)))


def test_zeros_infinities_and_nan():
    zero = [torch.zeros(5000, device=DEV), torch.zeros(3, dtype=BF16, device=DEV)]
    norm, norms = norm_of(zero)
    assert float(norm) == 0.0 and bool((norms == 0).all())
    for bad, check in ((math.inf, math.isinf), (-math.inf, math.isinf), (math.nan, math.isnan)):
        for t in (F32, BF16, F16):
            grads = tensors([500, 40000, 9], [t])
            grads[1][33333] = bad
            norm, norms = norm_of(grads)
            assert check(float(norm)) and check(float(norms[1])) and math.isfinite(float(norms[0])) and math.isfinite(float(norms[2]))
            before = [g.clone() for g in grads]
            out = torch.empty(1, device=DEV)
            gk.gk_grad_clip(grads, 0.5, norm_out=out)      # nothing is clipped
            assert check(float(out)) and gk.gk_grad_last_info() == (0, False)
            assert all(torch.equal(a.view(torch.int16 if t != F32 else torch.int32), b.view(torch.int16 if t != F32 else torch.int32)) for a, b in zip(grads, before))


def test_no_tensors():
    norm = torch.full((1,), -7.0, device=DEV)
    gk.gk_grad_norm([], norm, norms_out=torch.empty(0, device=DEV))
    assert float(norm) == 0.0
    norm.fill_(-7.0)
    gk.gk_grad_clip([], 1.0, norm_out=norm)
    assert float(norm) == 0.0 and gk.gk_grad_last_info() == (0, False)


@pytest.mark.parametrize("types", [[F32], [BF16], [F16], [F32, BF16, F16]], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("name", LISTS)
def test_clipping_into_the_sparsifiers_vector(name, types):
    grads = tensors(LISTS[name], types, seed=len(name) + 1)
    total = float(norms64(grads).square().sum().sqrt())
    n = sum(g.numel() for g in grads)
    for share in (0.3, 2.0):
        store = torch.full((n + 4,), -7.0, device=DEV)
        norm = torch.empty(1, device=DEV)
        gk.gk_grad_clip(grads, share * total, out=store[:n], norm_out=norm)
        assert bool((store[n:] == -7).all())
        check_norms(grads, norm)
        check_clipped(grads, torch.split(store[:n], [g.numel() for g in grads]), share * total)
        assert gk.gk_grad_last_info() == (0, share < 1)


@pytest.mark.parametrize("shift,out_shift", [(0, 0), (1, 1), (1, 3), (0, 5)])
@pytest.mark.parametrize("src", [F32, BF16, F16])
@pytest.mark.parametrize("dst", [F32, BF16, F16])
def test_clipping_into_other_tensors(src, dst, shift, out_shift):
    sizes = [1, 15, 4096, 0, 50001]
    grads, outs = tensors(sizes, [src], shift=shift), tensors(sizes, [dst], seed=9, shift=out_shift)
    before = [g.clone() for g in grads]
    limit = 0.4 * float(norms64(grads).square().sum().sqrt())
    gk.gk_grad_clip(grads, limit, out=outs)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    check_clipped(before, outs, limit)
    for o, n in zip(outs, sizes):      # what lies around an output stays
        assert bool((torch.as_strided(o, (3,), (1,), o.storage_offset() + n) == 7).all())
        assert out_shift == 0 or bool((torch.as_strided(o, (out_shift,), (1,), 0) == 7).all())


@pytest.mark.parametrize("types", [[F32], [BF16], [F32, BF16, F16]], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("shift", [0, 3])
def test_clipping_in_place(types, shift):
    grads = tensors([70001, 3, 0, 4096, 12345], types, shift=shift)
    before = [g.clone() for g in grads]
    total = float(norms64(grads).square().sum().sqrt())
    gk.gk_grad_clip(grads, 2.0 * total)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    gk.gk_grad_clip(grads, 0.25 * total)
    check_clipped(before, grads, 0.25 * total)


def test_a_norm_and_a_scale_that_the_caller_has():
    grads = tensors([30001, 64], [F16], scale=10.0)
    before = [g.clone() for g in grads]
    total = float(norms64(grads).square().sum().sqrt())
    scale, norm = torch.full((1,), 2.0 ** -7, device=DEV), torch.empty(1, device=DEV)
    out = torch.empty(30065, device=DEV)
    gk.gk_grad_clip(grads, 0.5 * total / 128, out=out, scale=scale, norm_out=norm)
    assert abs(float(norm) - total / 128) <= NORM_TOL * total / 128
    check_clipped(before, torch.split(out, [30001, 64]), 0.5 * total / 128, scale=2.0 ** -7)
    # as if other ranks held as much again
    given = torch.full((1,), 3.0, device=DEV)
    gk.gk_grad_clip(grads, 1.5, out=out, norm_in=given, norm_out=norm)
    assert float(norm) == 3.0 and gk.gk_grad_last_info() == (0, True)
    check_clipped(before, torch.split(out, [30001, 64]), 1.5, norm=3.0)
    scale.fill_(-0.5)
    gk.gk_grad_clip(grads, math.inf, scale=scale)
    check_clipped(before, grads, math.inf, scale=-0.5)


def test_a_norm_beyond_fp32_clips_nothing():
    for g in (torch.full((2000,), 3e38, device=DEV), torch.full((70000,), 3e38, dtype=BF16, device=DEV)):
        before, norm, out = g.clone(), torch.empty(1, device=DEV), torch.zeros(g.numel(), device=DEV)
        gk.gk_grad_clip([g], 1.0, out=out, norm_out=norm)
        assert math.isinf(float(norm)) and gk.gk_grad_last_info() == (0, False) and torch.equal(out, before.float())
        gk.gk_grad_clip([g], 1.0, norm_in=norm)
        assert torch.equal(g, before)
        # within fp32 once scaled
        scale = torch.full((1,), 2.0 ** -40, device=DEV)
        gk.gk_grad_clip([g], 2.0 ** 20, scale=scale, norm_out=norm)
        check_norms([before.double() * 2.0 ** -40], norm)
        check_clipped([before], [g], 2.0 ** 20, scale=2.0 ** -40)


def test_offsets_past_32_bits():
    n = (1 << 32) + 4099
    g = torch.zeros(n, dtype=BF16, device=DEV)
    g[-5000:] = 0.5
    g[:3] = 2.0
    norm = torch.empty(1, device=DEV)
    small = torch.ones(100, device=DEV)
    gk.gk_grad_norm([small, g], norm)
    want = math.sqrt(100 + 5000 * 0.25 + 12)
    assert abs(float(norm) - want) <= NORM_TOL * want
    gk.gk_grad_clip([small, g], want / 2, norm_out=norm)
    assert float(small[0]) == 0.5 and bool((g[-5000:] == 0.25).all()) and bool((g[:3] == 1.0).all()) and float(g[-5001]) == 0.0


def test_the_same_call_gives_the_same_bits_and_replays():
    grads = tensors([1_000_003, 77, 300_000], [BF16, F32])
    limit = 0.5 * float(norms64(grads).square().sum().sqrt())
    out, norm = torch.empty(1_300_080, device=DEV), torch.empty(1, device=DEV)
    gk.gk_grad_clip(grads, limit, out=out, norm_out=norm)
    first = out.clone(), norm.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        gk.gk_reserve(1, 1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            gk.gk_grad_clip(grads, limit, out=out, norm_out=norm)
    for scale in (1.0, 3.0, 0.125):
        for g in grads:
            g.mul_(scale)
        torch.cuda.synchronize()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if scale == 1.0:
            assert torch.equal(out, first[0]) and torch.equal(norm, first[1])
        check_norms(grads, norm)
        check_clipped(grads, torch.split(out, [g.numel() for g in grads]), limit)


def test_a_barrier_that_never_completes_is_given_up():
    grads = tensors([200_000, 5000], [F32])
    before = [g.clone() for g in grads]
    norm = torch.empty(1, device=DEV)
    gk.gk_debug_set(gk.KNOB_EXTRA_ARRIVALS, 1)
    gk.gk_debug_set(gk.KNOB_BARRIER_POLLS, 1000)
    try:
        gk.gk_grad_clip(grads, 1e-3, norm_out=norm)
        assert gk.gk_grad_last_info()[0] & gk.GK_DEV_TIMEOUT
        assert math.isnan(float(norm)) and all(torch.equal(a, b) for a, b in zip(grads, before))
    finally:
        gk.gk_debug_set(gk.KNOB_EXTRA_ARRIVALS, 0)
        gk.gk_debug_set(gk.KNOB_BARRIER_POLLS, 1 << 24)
    gk.gk_grad_clip(grads, 1e-3, norm_out=norm)
    assert gk.gk_grad_last_info() == (0, True)
    check_clipped(before, grads, 1e-3)


def test_refusals():
    g = [torch.zeros(8, device=DEV), torch.zeros(5, dtype=BF16, device=DEV)]
    one = torch.zeros(1, device=DEV)
    for bad in ([g[0].double()], [g[0].cpu()], [g[0][::2]], ["x"], [g[0].to(torch.int32)]):
        with pytest.raises(gk.GkError):
            gk.gk_grad_norm(bad, one)
        with pytest.raises(gk.GkError):
            gk.gk_grad_clip(bad, 1.0)
    for args, kw in (((g, one.double()), {}), ((g, torch.zeros(2, device=DEV)), {}), ((g, None), {}), ((g, one), {"norms_out": torch.zeros(3, device=DEV)})):
        with pytest.raises(gk.GkError):
            gk.gk_grad_norm(*args, **kw)
    big = torch.zeros(64, device=DEV)
    for args, kw in (((g, 0.0), {}), ((g, -1.0), {}), ((g, math.nan), {}), ((g, 1.0), {"out": torch.zeros(12, device=DEV)}),
                     ((g, 1.0), {"out": [g[0]]}), ((g, 1.0), {"out": [g[0], torch.zeros(6, device=DEV)]}),
                     ((g, 1.0), {"norm_out": one.double()}), ((g, 1.0), {"scale": 1.0}),
                     (([g[0], g[0]], 1.0), {}),                                           # in place twice
                     (([big[:8], big[4:12]], 1.0), {}),
                     (([big[:8]], 1.0), {"out": big[4:12]}),
                     (([big[:8], big[8:16]], 1.0), {"out": [big[8:16], big[:8]]}),        # each the other's
                     (([big[:8]], 1.0), {"out": [big.view(BF16)[:8]]}),
                     ((gk.GradList(g), 1.0), {"out": torch.zeros(13, device=DEV)})):
        with pytest.raises(gk.GkError):
            gk.gk_grad_clip(*args, **kw)
    # a tensor twice is fine where the outputs are others
    t = torch.ones(10, device=DEV)
    out = torch.empty(20, device=DEV)
    gk.gk_grad_clip([t, t], 1.0, out=out, norm_out=one)
    assert abs(float(one) - math.sqrt(20)) <= NORM_TOL * math.sqrt(20)
    check_clipped([t, t], [out[:10], out[10:]], 1.0)
