"""Host threads that call the vocabulary head on one stream: a call is several launches over the stream's
workspace, and each result is, bit by bit, that of the same call by a lone thread."""
import threading

import pytest
import torch

from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PER_THREAD = 2      # the handle of the calling thread's own default stream


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


class Work:
    """One thread's inputs, and its calls with result buffers of their own."""

    def __init__(self, seed, n, D, V, K=0):
        gen = torch.Generator().manual_seed(seed)
        self.n, self.D, self.V, self.K = n, D, V, K
        self.h = torch.randn(n, D, generator=gen).bfloat16().to(DEV)
        self.w = (torch.randn(V, D, generator=gen) / 8).bfloat16().to(DEV)
        self.target = torch.randint(-1, V, (n,), generator=gen).to(DEV)       # some rows left out
        if K:
            self.idx = torch.stack([torch.randperm(V, generator=gen)[:K].sort().values for _ in range(n)]).to(torch.int32).to(DEV)
            self.val = torch.randn(n, K, generator=gen).to(DEV)

    def outputs(self):
        return torch.empty(self.n, device=DEV), torch.empty(self.n, device=DEV), torch.empty_like(self.h), torch.empty_like(self.w)

    def call(self, out):
        loss, lse, dh, dw = out
        if self.K:
            gk.gk_vocab_distill(self.h, self.w, self.idx, self.val, loss, lse, dh=dh, dw=dw)
        else:
            gk.gk_vocab_loss(self.h, self.w, self.target, loss, lse, dh=dh, dw=dw)

    def call_on(self, stream, out):
        """The same through the C interface, on any stream handle."""
        loss, lse, dh, dw = (x.data_ptr() for x in out)
        return gk.load().gk_vocab_loss(self.h.data_ptr(), self.D, self.w.data_ptr(), self.D, 1, self.n, self.D, self.V, self.target.data_ptr(),
                                       -1, None, loss, lse, dh, self.D, dw, self.D, stream)


def together(threads):
    failed = []
    gate = threading.Barrier(len(threads))

    def body(f):
        try:
            gate.wait()
            f()
        except Exception as e:      # noqa: BLE001
            failed.append(e)

    run = [threading.Thread(target=body, args=(f,)) for f in threads]
    for t in run:
        t.start()
    for t in run:
        t.join()
    assert not failed, failed


def expect(work, outs):
    want = work.outputs()
    torch.cuda.synchronize()
    work.call(want)
    torch.cuda.synchronize()
    for out in outs:
        for a, b in zip(out, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("reserved", [True, False])
def test_two_threads_on_one_stream(reserved):
    """Not reserved: the threads' calls also replace the workspace, each growing it beyond what it was."""
    stream = torch.cuda.Stream()
    works = [Work(1, 300, 200, 1500), Work(2, 280, 136, 2100, K=9), Work(3, 1200, 64, 900)]
    outs = [[w.outputs() for _ in range(12)] for w in works]
    if reserved:
        with torch.cuda.stream(stream):
            for w in works:
                gk.gk_vocab_reserve(w.n, w.D, w.V, max(1, w.K))
    torch.cuda.synchronize()

    def body(w, mine):
        with torch.cuda.stream(stream):
            for out in mine:
                w.call(out)

    together([lambda w=w, mine=mine: body(w, mine) for w, mine in zip(works, outs)])
    torch.cuda.synchronize()
    for w, mine in zip(works, outs):
        expect(w, mine)


def test_the_per_thread_streams_have_a_workspace_each():
    works = [Work(4, 300, 200, 1500), Work(5, 300, 200, 1500)]
    outs = [[w.outputs() for _ in range(12)] for w in works]
    torch.cuda.synchronize()

    def body(w, mine):
        torch.cuda.set_device(0)
        for out in mine:
            assert w.call_on(PER_THREAD, out) == 0

    together([lambda w=w, mine=mine: body(w, mine) for w, mine in zip(works, outs)])
    torch.cuda.synchronize()
    for w, mine in zip(works, outs):
        expect(w, mine)


def test_a_reader_of_the_last_call_beside_callers():
    stream = torch.cuda.Stream()
    work = Work(6, 300, 200, 1500)
    outs = [work.outputs() for _ in range(12)]
    rows = int((work.target >= 0).sum())
    with torch.cuda.stream(stream):
        gk.gk_vocab_reserve(work.n, work.D, work.V)
        work.call(outs[0])
    torch.cuda.synchronize()

    def calls():
        with torch.cuda.stream(stream):
            for out in outs:
                work.call(out)

    def reads():
        with torch.cuda.stream(stream):
            for _ in range(12):
                status, counted = gk.gk_vocab_last_info()
                assert status == 0 and counted == rows

    together([calls, reads])
    torch.cuda.synchronize()
    expect(work, outs)
