"""What the vocabulary head's calls refuse on the host, beyond the sizes, types and pointers of the library's interface test."""
import pytest

from paper_1911_08772_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


@pytest.mark.parametrize("T", [1e-40, 1e-45, 4e-39])
def test_a_temperature_without_a_reciprocal(lib, T):
    """Equal logits were divided by it into infinity times zero."""
    a = 0x100000
    assert lib.gk_vocab_topk(a, 50, 0, 2, 50, 4, T, a, a, None, None) == -12
    assert lib.gk_vocab_distill(a, 8, a + 0x10000, 8, 1, 4, 8, 5, a, a, 3, None, T, None, a, a, None, 8, None, 8, None) == -12
    assert "temperature" in binding.gk_strerror(-12)
