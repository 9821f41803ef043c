"""What gk_grad_norm and gk_grad_clip refuse on the host, before they touch a device."""
import ctypes as C

import pytest

from paper_1911_08772_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def lists(pointers, types, sizes):
    n = len(pointers)
    return (C.c_void_p * n)(*pointers), (C.c_int32 * n)(*types), (C.c_int64 * n)(*sizes)


A = 0x100000


@pytest.mark.parametrize("pointers,types,sizes,want", [
    ([A], [3], [8], -10), ([A], [-1], [8], -10), ([A], [0], [-1], -2), ([None], [0], [8], -1), ([A + 2], [0], [8], -4),
    ([A + 1], [1], [8], -4), ([A], [0], [2 ** 44 + 1], -9)])
def test_lists(lib, pointers, types, sizes, want):
    p, t, n = lists(pointers, types, sizes)
    assert lib.gk_grad_norm(p, t, n, len(pointers), A, None, None) == want
    assert lib.gk_grad_clip(p, t, p, t, n, len(pointers), 1.0, None, None, None, None) == want


def test_the_rest(lib):
    p, t, n = lists([A, A + 64], [0, 0], [16, 16])
    assert lib.gk_grad_norm(p, t, n, 2, None, None, None) == -1
    assert lib.gk_grad_norm(None, t, n, 2, A, None, None) == -1
    assert lib.gk_grad_norm(p, t, n, -1, A, None, None) == -2
    assert lib.gk_grad_norm(p, t, n, 65537, A, None, None) == -9
    assert lib.gk_grad_clip(p, t, None, t, n, 2, 1.0, None, None, None, None) == -1
    assert lib.gk_grad_clip(p, t, p, None, n, 2, 1.0, None, None, None, None) == -1
    for norm in (0.0, -1.0, float("nan")):
        assert lib.gk_grad_clip(p, t, p, t, n, 2, norm, None, None, None, None) == -13
    clip = lambda src, dst, types=(0, 0), out_types=(0, 0): lib.gk_grad_clip(  # noqa: E731
        *lists(src, types, [16, 16])[:2], *lists(dst, out_types, [16, 16]), 2, 1.0, None, None, None, None)
    assert clip([A, A + 64], [A, A + 60]) == -5                  # outputs that overlap
    assert clip([A, A + 64], [A + 64, A]) == -5                  # each the other's input
    assert clip([A, A], [A, A]) == -5                            # in place twice
    assert clip([A, A + 64], [A, A + 64], out_types=(1, 0)) == -5     # in place as another type
    assert clip([A, A + 640], [A + 4, A + 6400]) == -5
    assert clip([A, A + 640], [A + 6400, A + 640 + 60]) == -5
    assert clip([A, A + 64], [A + 6400, A + 64002]) == -4
    assert clip([A, A + 64], [A + 6400, None]) == -1
    assert clip([A, A + 64], [A + 6400, A + 64000], out_types=(0, 7)) == -10
    assert "norm" in binding.gk_strerror(-13)
    out = (C.c_int64 * 2)()
    assert lib.gk_grad_last_info(None, None) == -1
