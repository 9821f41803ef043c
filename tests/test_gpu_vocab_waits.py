"""Every wait in the products of the vocabulary head is bounded: readers that wait for sums which never
arrive give up, so do the warps that then wait for the readers, the call ends with GK_DEV_TIMEOUT in
its status word, and the next call is right.  The wait is made to run out by a barrier that expects one
arrival more than there are; nothing hangs and nothing faults."""
import pytest
import torch

from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield
    gk.gk_debug_set(gk.KNOB_EXTRA_ARRIVALS, 0)


@pytest.mark.parametrize("n,D,V", [(40, 64, 300), (300, 1600, 5000)])
def test_readers_whose_sums_never_arrive_give_up(n, D, V):
    gen = torch.Generator().manual_seed(1)
    h, w = torch.randn(n, D, generator=gen).bfloat16().to(DEV), (torch.randn(V, D, generator=gen) / 8).bfloat16().to(DEV)
    target = torch.randint(0, V, (n,), generator=gen).to(DEV)

    def call():
        loss, lse, dh, dw = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty_like(h), torch.empty_like(w)
        gk.gk_vocab_loss(h, w, target, loss, lse, dh=dh, dw=dw)
        return loss, lse, dh, dw, gk.gk_vocab_last_info()

    good = call()
    assert good[4] == (0, n)
    gk.gk_debug_set(gk.KNOB_EXTRA_ARRIVALS, 1)
    assert call()[4][0] & gk.GK_DEV_TIMEOUT
    gk.gk_debug_set(gk.KNOB_EXTRA_ARRIVALS, 0)
    again = call()
    assert again[4] == (0, n)
    for a, b in zip(good[:4], again[:4]):
        assert torch.equal(a, b)
