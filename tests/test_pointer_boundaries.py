"""Every pointer of the vocabulary's and the gradients' calls off its type's boundary is refused on the host: a kernel
would fault on it."""
import ctypes as C

import pytest

from paper_1911_08772_b200 import binding, build

A, B = 0x1000000, 0x2000000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def grad_lists():
    return (C.c_void_p * 1)(A), (C.c_int32 * 1)(0), (C.c_int64 * 1)(8)


# name: (the call's arguments, what is at which place: bytes of its boundary)
def calls():
    g, t, s = grad_lists()
    return {
        "gk_vocab_logprob": ([A, 50, 0, 2, 50, B, 1, 1.0, 4, B, B, B, B, B, B, None], {5: 8, 9: 4, 10: 4, 11: 4, 12: 4, 13: 4, 14: 4}),
        "gk_vocab_logprob_grad": ([A, 50, 0, 2, 50, B, 1, 1.0, B, B, B, B, B, B, 50, None], {5: 8, 8: 4, 9: 4, 10: 4, 11: 4, 12: 4}),
        "gk_vocab_topk": ([A, 50, 0, 2, 50, 4, 1.0, B, B, B, None], {7: 4, 8: 4, 9: 4}),
        "gk_vocab_loss": ([A, 8, A + 0x10000, 8, 1, 4, 8, 50, B, -100, B, B, B, None, 8, None, 8, None], {8: 8, 10: 4, 11: 4, 12: 4}),
        "gk_vocab_distill": ([A, 8, A + 0x10000, 8, 1, 4, 8, 50, B, B, 3, B, 1.0, B, B, B, None, 8, None, 8, None],
                             {8: 4, 9: 4, 11: 4, 13: 4, 14: 4, 15: 4}),
        "gk_grad_norm": ([g, t, s, 1, B, B, None], {4: 4, 5: 4}),
        "gk_grad_clip": ([g, t, g, t, s, 1, 1.0, B, B + 64, B + 128, None], {7: 4, 8: 4, 9: 4}),
    }


@pytest.mark.parametrize("name", ["gk_vocab_logprob", "gk_vocab_logprob_grad", "gk_vocab_topk", "gk_vocab_loss", "gk_vocab_distill", "gk_grad_norm", "gk_grad_clip"])
def test_pointers_off_their_boundaries(lib, name):
    args, places = calls()[name]
    for at, size in places.items():
        for by in (1, 2, 4):
            if by < size:
                assert getattr(lib, name)(*args[:at], args[at] + by, *args[at + 1:]) == -4, (at, by)
