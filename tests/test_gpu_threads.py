"""Host threads that call the sparsifiers on one stream, with vectors of different lengths that grow the
stream's workspace under one another: each result is, bit by bit, that of the same call by a lone thread."""
import threading

import numpy as np
import pytest
import torch

from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PER_THREAD = 2      # the handle of the calling thread's own default stream


@pytest.fixture(autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    gk.gk_set_path(0)
    gk.gk_set_capacity(0)
    yield
    gk.gk_set_path(0)


class Steps:
    """One thread's error-compensated steps on vectors of d elements, and Top_k of the last."""

    def __init__(self, seed, d, steps=6):
        gen = torch.Generator().manual_seed(seed)
        self.d, self.k = d, max(1, d // 500)
        self.g = [(torch.randn(d, generator=gen) * 1e-2).to(DEV) for _ in range(steps)]
        self.clear()

    def clear(self):
        self.eps = torch.zeros(self.d, device=DEV)
        self.out = [(torch.full((self.d,), -1, dtype=torch.int32, device=DEV), torch.zeros(self.d, device=DEV),
                     torch.zeros(1, dtype=torch.int64, device=DEV)) for _ in self.g]
        self.top = torch.empty(self.k, dtype=torch.int32, device=DEV), torch.empty(self.k, device=DEV)

    def run(self, stream):
        L = gk.load()
        torch.cuda.set_device(0)
        for g, (idx, val, nnz) in zip(self.g, self.out):
            assert L.gk_sparsify(g.data_ptr(), self.eps.data_ptr(), self.d, self.k, idx.data_ptr(), val.data_ptr(), nnz.data_ptr(), stream) == 0
        assert L.topk_exact(self.g[-1].data_ptr(), self.d, self.k, self.top[0].data_ptr(), self.top[1].data_ptr(), stream) == 0

    def results(self):
        torch.cuda.synchronize()
        got = [self.eps, *self.top]
        for idx, val, nnz in self.out:
            n = int(nnz)
            got += [idx[:n], val[:n], nnz]
        return [x.cpu().numpy().copy() for x in got]


@pytest.mark.parametrize("path", [0, 1, 2])
@pytest.mark.parametrize("per_thread", [False, True])
def test_threads_on_one_stream(per_thread, path):
    """Paths: 0 as chosen by size, 1 the three kernels, 2 the persistent kernel."""
    gk.gk_set_path(path)
    works = [Steps(1, 70001), Steps(2, 1300003), Steps(3, 2500000)]
    alone = []
    for w in works:
        torch.cuda.synchronize()
        w.run(torch.cuda.Stream().cuda_stream)
        alone.append(w.results())
        w.clear()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    failed, gate = [], threading.Barrier(len(works))

    def body(w):
        try:
            gate.wait()
            w.run(PER_THREAD if per_thread else stream.cuda_stream)
        except BaseException as e:      # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=body, args=(w,)) for w in works]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for w, want in zip(works, alone):
        for a, b in zip(w.results(), want):
            assert np.array_equal(a, b)
