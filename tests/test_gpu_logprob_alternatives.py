"""gk_vocab_logprob's most probable tokens where the first words of a row say little of the rest: masks over parts of the
vocabulary, so that fewer logits than are asked for come above the threshold that those words give."""
import math

import pytest
import torch

from logprob_util import logp_tol
from paper_1911_08772_b200 import binding as gk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1911_08772_b200 import build
    build.build()
    gk.load()
    yield


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("k", [1, 20, 100, 128])
@pytest.mark.parametrize("n,V", [(686, 5827), (160, 1003), (152, 26289), (228, 17486), (40, 71795), (3, 128000), (20, 9001)])
def test_alternatives_of_rows_masked_in_parts(n, V, k, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + k)
    for mask in (-math.inf, -1e4, -60000.0):
        for begin, end in ((0.1, 1.0), (0.0, 0.9), (0.03, 0.6), (0.26, 0.99)):
            z = torch.randn(n, V, generator=gen, device=DEV) * 3
            z[:, int(begin * V):int(end * V)] = mask
            z = z.to(dtype)
            idx = torch.full((n, k), -7, dtype=torch.int32, device=DEV)
            val, lse = torch.full((n, k), -7.0, device=DEV), torch.empty(n, device=DEV)
            gk.gk_vocab_logprob(z, None, lse_out=lse, idx_out=idx, val_out=val)
            want = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :k]
            assert torch.equal(idx.long(), want), (mask, begin, end)
            logp = torch.log_softmax(z.double(), 1).gather(1, want)
            fine = logp > -math.inf
            off = (torch.where(fine, val.double() - logp, 0.0)).abs().cpu()
            assert bool((off <= logp_tol(torch.where(fine, logp, 0.0).cpu())).all()) and bool((val[~fine] == -math.inf).all())
