"""What gk_vocab_logprob and gk_vocab_logprob_grad refuse on the host, before they touch a device."""
import pytest

from paper_1911_08772_b200 import binding, build

A, B = 0x1000000, 0x2000000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def forward(lib, logits=A, ld=50, dtype=0, n=2, V=50, token=B, m=1, T=1.0, k=4, idx=B, val=B):
    return lib.gk_vocab_logprob(logits, ld, dtype, n, V, token, m, T, k, B, B, B, B, idx, val, None)


def backward(lib, logits=A, ld=50, dtype=0, n=2, V=50, token=B, m=1, T=1.0, lse=B, entropy=B, b=B, dz=B, lddz=50):
    return lib.gk_vocab_logprob_grad(logits, ld, dtype, n, V, token, m, T, lse, entropy, B, b, None, dz, lddz, None)


@pytest.mark.parametrize("change,want", [
    ({"n": -1}, -2), ({"V": 0}, -2), ({"V": 2 ** 31, "ld": 2 ** 31}, -2), ({"m": -1}, -2), ({"m": 129}, -9), ({"n": 2 ** 31}, -9),
    ({"dtype": 3}, -10), ({"logits": None}, -1), ({"token": None}, -1), ({"ld": 49}, -11), ({"logits": A + 2}, -4),
    ({"logits": A + 1, "dtype": 1}, -4), ({"T": 0.0}, -12), ({"T": -1.0}, -12), ({"T": float("nan")}, -12), ({"T": float("inf")}, -12), ({"T": 1e-40}, -12)])
def test_both(lib, change, want):
    assert forward(lib, **change) == want
    assert backward(lib, **change) == want


@pytest.mark.parametrize("change,want", [({"k": -1}, -3), ({"k": 51}, -3), ({"k": 129, "V": 500, "ld": 500}, -3), ({"idx": None}, -1), ({"val": None}, -1)])
def test_alternatives(lib, change, want):
    assert forward(lib, **change) == want


@pytest.mark.parametrize("change,want", [
    ({"lse": None}, -1), ({"dz": None}, -1), ({"entropy": None}, -1), ({"lddz": 49}, -11), ({"dz": B + 2}, -4), ({"dz": A + 4}, -5),
    ({"dz": A, "lddz": 51}, -5), ({"dz": A + 396}, -5), ({"logits": A, "dz": A - 4}, -5)])
def test_gradients(lib, change, want):
    assert backward(lib, **change) == want


def test_no_rows(lib):
    assert forward(lib, n=0, logits=None, token=None, idx=None, val=None) == 0
    assert backward(lib, n=0, logits=None, token=None, lse=None, dz=None, entropy=None) == 0


def test_rows_between_rows(lib):
    """Rows of 50 floats, 103 apart: gradients 50 to 53 elements on lie between the logits, any others that begin among
    them do not."""
    for by in (1, 49, 54, 102, 103, 103 + 49, 103 + 54):
        assert backward(lib, n=4, ld=103, lddz=103, dz=A + 4 * by) == -5
        assert backward(lib, n=4, ld=103, lddz=103, logits=A + 4 * by, dz=A) == -5
    assert backward(lib, n=4, ld=103, lddz=104, dz=A + 4 * 51) == -5
