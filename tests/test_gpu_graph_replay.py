"""Calls captured in a graph and replayed on new data: each replay gives what an eager call gives."""
import numpy as np
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
    gk.gk_set_path(0)
    gk.gk_set_capacity(0)
    yield
    gk.gk_set_path(0)


CALLS = ["gk_sparsify_static", "gk_sparsify", "gk_select", "topk_exact", "topk_sparsify"]


# by path: 0 as chosen by size, 2 the persistent kernel, 1 the kernels of several launches (gk_sparsify_static has the second alone)
CASES = [(c, p, d) for c in CALLS for p, d in ((0, 300007), (2, 300007), (1, 300007), (0, 2500000)) if p != 1 or c != "gk_sparsify_static"]


@pytest.mark.parametrize("call,path,d", CASES)
def test_replays_on_new_data(call, path, d):
    """The scale changes by 100 from replay to replay, so that a replay with anything of the one before selects
    other elements."""
    gk.gk_set_path(path)
    L = gk.load()
    gen = torch.Generator().manual_seed(d + path)
    k = d // 1000
    data = [(torch.randn(d, generator=gen) * (1e-4 if i % 2 else 1e-2)).to(DEV) for i in range(8)]
    g, eps = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    idx, val = torch.empty(d, dtype=torch.int32, device=DEV), torch.empty(d, device=DEV)
    nnz = torch.zeros(1, dtype=torch.int64, device=DEV)
    stream = torch.cuda.Stream()

    def enqueue(st):
        p = [x.data_ptr() for x in (g, eps, idx, val, nnz)]
        if call in ("gk_sparsify_static", "gk_sparsify", "topk_sparsify"):
            rc = getattr(L, call)(p[0], p[1], d, k, p[2], p[3], p[4], st)
        elif call == "gk_select":
            rc = L.gk_select(p[0], d, k, p[2], p[3], p[4], st)
        else:
            rc = L.topk_exact(p[0], d, k, p[2], p[3], st)
        assert rc == 0

    def results(x, run):
        g.copy_(x)
        eps.zero_()
        idx.fill_(-1)
        val.zero_()
        nnz.fill_(k)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        n = int(nnz)
        return [t.cpu().numpy().copy() for t in (idx[:n], val[:n], eps)]

    with torch.cuda.stream(stream):
        eager = [results(x, lambda: enqueue(stream.cuda_stream)) for x in data]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            enqueue(torch.cuda.current_stream().cuda_stream)
        for x, want in zip(data, eager):
            for a, b in zip(results(x, graph.replay), want):
                assert np.array_equal(a, b)
