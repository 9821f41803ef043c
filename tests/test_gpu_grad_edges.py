"""gk_grad_clip where its bounded wait runs out for some of its CTAs, and its scalars' places."""
import math

import pytest
import torch

from grad_util import NORM_TOL, check_clipped, tensors
from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


def test_all_of_a_grid_or_none_of_it_gives_up():
    """Waits that give up at the first look: some CTAs would, and those that arrive last would not.  Either nothing is
    written and the norm is NaN, or the call is whole."""
    grads = tensors([1_200_000, 70_001, 5000], [F32, BF16])
    before = [g.clone() for g in grads]
    norm = torch.empty(1, device=DEV)
    gave_up = 0
    try:
        for polls in [0] * 100 + [1] * 30 + [3] * 30 + [10] * 40:
            gk.gk_debug_set(gk.KNOB_BARRIER_POLLS, polls)
            norm.fill_(-7.0)
            gk.gk_grad_clip(grads, 1e-3, norm_out=norm)
            flags, clipped = gk.gk_grad_last_info()
            if flags:
                gave_up += 1
                assert flags == gk.GK_DEV_TIMEOUT and not clipped and math.isnan(float(norm))
                assert all(torch.equal(a, b) for a, b in zip(grads, before))
            else:
                assert clipped and float(norm) > 0
                check_clipped(before, grads, 1e-3)
                for a, b in zip(grads, before):
                    a.copy_(b)
    finally:
        gk.gk_debug_set(gk.KNOB_BARRIER_POLLS, 1 << 24)
    assert gave_up > 0
    gk.gk_grad_clip(grads, 1e-3, norm_out=norm)
    assert gk.gk_grad_last_info() == (0, True)
    check_clipped(before, grads, 1e-3)


def test_a_norm_where_a_scalar_was():
    grads = tensors([300_000, 5000], [F32])
    before = [g.clone() for g in grads]
    total = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    one = torch.full((1,), 2.0, device=DEV)
    gk.gk_grad_clip(grads, 1.0, norm_in=one, norm_out=one)
    assert float(one) == 2.0
    check_clipped(before, grads, 1.0, norm=2.0)
    for g, b in zip(grads, before):
        g.copy_(b)
    gk.gk_grad_clip(grads, 0.5 * total, scale=one, norm_out=one)
    assert abs(float(one) - 2 * total) <= 2 * NORM_TOL * total
    check_clipped(before, grads, 0.5 * total, scale=2.0)
    with pytest.raises(gk.GkError):
        gk.gk_grad_clip(grads, 1.0, scale=one, norm_in=torch.ones_like(one), norm_out=one)
    for kw in ({"scale": grads[1][:1]}, {"norm_in": grads[0][:1]}, {"norm_out": grads[0][7:8]}):
        with pytest.raises(gk.GkError):
            gk.gk_grad_clip(grads, 1.0, **kw)
