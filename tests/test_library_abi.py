"""Host-side checks of the C ABI that need no GPU: the library loads, exports every
symbol include/gk.h declares, and rejects bad arguments before touching the device."""
import ctypes as C
import os
import re

import pytest

from paper_1911_08772_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def declared_functions():
    text = open(os.path.join(ROOT, "include", "gk.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = re.findall(r"\b([a-z_0-9]+)\s*\(", text)
    return sorted({n for n in names if n.startswith(("gk_", "topk_", "dgck_"))})


def test_every_declared_symbol_is_exported(lib):
    names = declared_functions()
    assert set(binding.EXPORTS) <= set(names)
    for n in ("gk_sparsify", "gk_sparsify_segmented", "topk_exact"):
        assert n in names
    for n in names:
        assert hasattr(lib, n), n


def test_version_and_error_text(lib):
    assert lib.gk_version() >= 1000
    assert binding.gk_strerror(0) == "ok"
    for code in range(-9, 0):
        assert "unknown" not in binding.gk_strerror(code)
    assert "unknown" in binding.gk_strerror(-99)


def test_workspace_bytes_is_modest_and_monotone(lib):
    small = binding.gk_workspace_bytes(1, 1)
    big = binding.gk_workspace_bytes(1 << 28, 1)
    seg = binding.gk_workspace_bytes(25_557_032, 161)
    assert 0 < small <= big
    assert big < 8 << 20          # status words: 8 B per 8192-element tile
    assert seg < 8 << 20
    assert binding.gk_workspace_bytes(0, 1) == 0


def test_argument_validation_happens_on_the_host(lib):
    a = 0x1000  # a fake, aligned, non-null address: validation must fail before any use
    st = None
    assert lib.gk_sparsify(None, a, 10, 1, a, a, a, st) == -1
    assert lib.gk_sparsify(a, a + 4096, 0, 1, a, a, a, st) == -2
    assert lib.gk_sparsify(a, a + 4096, 2 ** 31, 1, a, a, a, st) == -2
    assert lib.gk_sparsify(a, a + 4096, 10, 0, a, a, a, st) == -3
    assert lib.gk_sparsify(a, a + 4096, 10, 11, a, a, a, st) == -3
    assert lib.gk_sparsify(a + 4, a + 4096, 10, 1, a, a, a, st) == -4
    assert lib.gk_sparsify(a, a + 16, 10, 1, a, a, a, st) == -5     # g overlaps eps
    assert lib.topk_exact(None, 10, 1, a, a, st) == -1
    assert lib.topk_exact(a, 10, 11, a, a, st) == -3
    assert lib.topk_exact(a + 8, 10, 1, a, a, st) == -4
    assert lib.gk_sparsify_segmented(a, a + 4096, 10, None, a, 1, a, a, None, a, st) == -1
    assert lib.gk_sparsify_segmented(a, a + 4096, 10, a, a, 0, a, a, None, a, st) == -2
    assert lib.gk_sparsify_segmented(a, a + 4096, 10, a, a, 70000, a, a, None, a, st) == -2
    assert lib.topk_sparsify(a, a + 16, 10, 1, a, a, a, st) == -5
    import ctypes
    out = (ctypes.c_double * 3)()
    assert lib.gk_error_ratio(None, 10, a, a, st, out) == -1
    assert lib.gk_error_ratio(a, 10, a, a, st, None) == -1
    assert lib.gk_error_ratio(a, 0, a, a, st, out) == -2
    assert lib.gk_error_ratio(a + 4, 10, a, a, st, out) == -4
    assert lib.gk_set_capacity(-1) == -8
    assert lib.gk_set_capacity(0) == 0


def test_binding_refuses_cpu_tensors(lib):
    import torch
    t = torch.zeros(8)
    with pytest.raises(binding.GkError):
        binding.gk_sparsify(t, t.clone(), 1, torch.zeros(8, dtype=torch.int32), t.clone(),
                            torch.zeros(1, dtype=torch.int64))


def test_dgck_argument_validation_happens_on_the_host(lib):
    a = 0x1000
    st = None
    assert lib.dgck_select(None, 10, 1, a, 5, a, a, a, st) == -1
    assert lib.dgck_select(a, 10, 1, None, 5, a, a, a, st) == -1
    assert lib.dgck_select(a, 0, 1, a, 5, a, a, a, st) == -2
    assert lib.dgck_select(a, 10, 1, a, 0, a, a, a, st) == -2
    assert lib.dgck_select(a, 10, 11, a, 5, a, a, a, st) == -3
    assert lib.dgck_select(a + 4, 10, 1, a, 5, a, a, a, st) == -4
    assert lib.dgck_sparsify(a, a + 16, 10, 1, a, 5, a, a, a, st) == -5
    assert lib.dgck_sparsify(a, None, 10, 1, a, 5, a, a, a, st) == -1


def test_the_operator_and_the_setters_validate_on_the_host(lib):
    a = 0x1000
    assert lib.gk_select(None, 10, 1, a, a, a, None) == -1
    assert lib.gk_select(a, 0, 1, a, a, a, None) == -2
    assert lib.gk_select(a, 10, 11, a, a, a, None) == -3
    assert lib.gk_select(a + 4, 10, 1, a, a, a, None) == -4
    assert lib.gk_set_params(1, 0) == -2 and lib.gk_set_params(0, 5) == -2     # rounds outside 1 .. 4
    assert lib.gk_set_path(3) == -2 and lib.gk_set_path(-1) == -2
    assert lib.gk_debug_set(99, 0) == -2 and lib.gk_debug_set(-1, 0) == -2      # unknown keys
    assert lib.gk_debug_set(0, -2) == -2                                         # value out of range


def test_the_vocabulary_head_validates_on_the_host(lib):
    a, st = 0x100000, None

    def loss(h=a, ldh=8, w=a + 0x10000, ldw=8, dtype=1, n=4, D=8, V=5, target=a, loss_out=a, lse=a, dh=None, lddh=8, dw=None, lddw=8):
        return lib.gk_vocab_loss(h, ldh, w, ldw, dtype, n, D, V, target, -100, None, loss_out, lse, dh, lddh, dw, lddw, st)

    assert loss(n=-1) == -2 and loss(D=0) == -2 and loss(V=0) == -2
    assert loss(n=2 ** 22 + 1) == -9 and loss(D=2 ** 16 + 1) == -9 and loss(V=2 ** 26 + 1) == -9
    assert loss(dtype=0) == -10 and loss(dtype=7) == -10
    assert loss(h=None) == -1 and loss(w=None) == -1 and loss(target=None) == -1 and loss(loss_out=None) == -1 and loss(lse=None) == -1
    assert loss(ldh=7) == -11 and loss(ldw=7) == -11 and loss(dh=a + 0x20000, lddh=7) == -11 and loss(dw=a + 0x20000, lddw=7) == -11
    assert loss(h=a + 1) == -4 and loss(dw=a + 0x20001) == -4
    assert loss(dh=a + 8) == -5 and loss(dw=a + 0x10000 + 32) == -5 and loss(dh=a + 0x20000, dw=a + 0x20008) == -5

    def distill(K=3, T=1.0, idx=a, val=a):
        return lib.gk_vocab_distill(a, 8, a + 0x10000, 8, 1, 4, 8, 5, idx, val, K, None, T, None, a, a, None, 8, None, 8, st)

    assert distill(K=0) == -3 and distill(K=1025) == -3
    assert distill(T=0.0) == -12 and distill(T=float("nan")) == -12 and distill(T=float("inf")) == -12
    assert distill(idx=None) == -1 and distill(val=None) == -1

    def topk(z=a, ld=50, dtype=0, n=2, V=50, k=4, T=1.0, idx=a, val=a):
        return lib.gk_vocab_topk(z, ld, dtype, n, V, k, T, idx, val, None, st)

    assert topk(n=-1) == -2 and topk(V=0) == -2 and topk(dtype=3) == -10 and topk(z=None) == -1 and topk(idx=None) == -1
    assert topk(ld=49) == -11 and topk(z=a + 2) == -4 and topk(k=0) == -3 and topk(k=51) == -3 and topk(T=-1.0) == -12
    assert topk(n=0, z=None) == 0
    assert lib.gk_vocab_set_budget(-1) == -8


def test_error_text_of_the_vocabulary_head(lib):
    for code in (-10, -11, -12):
        assert "unknown" not in binding.gk_strerror(code)


def test_the_vocabulary_heads_workspace_is_bounded_by_the_budget(lib):
    base = binding.gk_vocab_workspace_bytes(8192, 4096, 128000)
    try:
        binding.gk_vocab_set_budget(64 << 20)
        small = binding.gk_vocab_workspace_bytes(8192, 4096, 128000)
        assert base - small > 1 << 30
        assert binding.gk_vocab_workspace_bytes(8192, 4096, 128000, grad=False) < small
    finally:
        binding.gk_vocab_set_budget(2 << 30)
    assert binding.gk_vocab_workspace_bytes(0, 64, 64) == 0
