"""What gk_grad_clip refuses of its scalars on the host, before it touches a device."""
import ctypes as C

import pytest

from paper_1911_08772_b200 import binding, build

A, S = 0x100000, 0x200000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def clip(lib, src, dst, scale=None, norm_in=None, norm_out=None):
    n = len(src)
    types, sizes = (C.c_int32 * n)(*[0] * n), (C.c_int64 * n)(*[16] * n)
    return lib.gk_grad_clip((C.c_void_p * n)(*src), types, (C.c_void_p * n)(*dst), types, sizes, n, 1.0, scale, norm_in, norm_out, None)


def test_scalars_that_share_memory(lib):
    apart, place = [A, A + 64], [A + 640, A + 704]
    for dst in (apart, place):
        assert clip(lib, apart, dst, scale=S, norm_in=S + 4, norm_out=S) == -5
        for at in (dst[0], dst[0] + 60, dst[1] + 4):
            assert clip(lib, apart, dst, scale=at) == -5
            assert clip(lib, apart, dst, norm_in=at) == -5
            assert clip(lib, apart, dst, norm_out=at) == -5
    # a gradient of which another CTA has still to read
    assert clip(lib, apart, place, norm_out=A + 4) == -5
    assert clip(lib, [], [], scale=S, norm_in=S + 4, norm_out=S) == -5
