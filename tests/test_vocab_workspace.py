"""The workspace that gk_vocab_reserve makes for n rows holds every call of fewer rows, although such a call can
need more: dh is split into more parts, and a piece of the vocabulary comes nearer to the budget."""
import pytest

from paper_1911_08772_b200 import binding as gk, build


@pytest.fixture(autouse=True)
def _library():
    build.build()
    gk.load()
    yield
    gk.gk_vocab_set_budget(2 << 30)


@pytest.mark.parametrize("D,V,rows", [(4096, 32000, [4096, 3585, 3000, 1024, 100, 1]), (8192, 32000, [2048, 1537, 1025, 257, 1]),
                                      (512, 128000, [8192, 8000, 7681, 4097, 1]), (136, 2100, [1300, 1025, 700, 64, 3])])
@pytest.mark.parametrize("budget", [2 << 30, 100 << 20, 1 << 20])
def test_fewer_rows_need_no_more(D, V, rows, budget):
    gk.gk_vocab_set_budget(budget)
    needs = [gk.gk_vocab_workspace_bytes(n, D, V) for n in rows]
    assert needs[-1] > 0
    assert needs == sorted(needs, reverse=True), list(zip(rows, needs))


def test_every_number_of_rows_up_to_a_thousand():
    needs = [gk.gk_vocab_workspace_bytes(n, 1024, 5000, 4) for n in range(1, 1100)]
    assert needs == sorted(needs)


def test_fewer_pairs_need_no_more_and_no_gradients_less():
    a, b, c = (gk.gk_vocab_workspace_bytes(2000, 512, 9000, K) for K in (1, 40, 1024))
    assert a <= b <= c
    assert gk.gk_vocab_workspace_bytes(2000, 512, 9000, 40, grad=False) < b
    small = [gk.gk_vocab_workspace_bytes(n, 512, 9000, 40, grad=False) for n in (1, 255, 256, 257, 2000)]
    assert small == sorted(small)
