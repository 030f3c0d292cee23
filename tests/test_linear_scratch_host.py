"""CPU: how much scratch aep_linear asks for, by the alignment of its operands."""

import ctypes
import os

import pytest

from paper_2505_08944_amd import _lib as L

AT = 1 << 20  # an address (never read): aligned


def _lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libaep.so not built (run __graft_entry__.build())")
    return L.lib()


def desc(m, n, k, fp8=False, ldx=None, ldw=None, ldy=None, out=L.AEP_BF16):
    return L.LinearDesc(m, n, k, L.AEP_BF16, L.AEP_FP8_E4M3 if fp8 else L.AEP_BF16, out, L.AEP_F32, out, 0, ldx or k,
                        ldw or k, ldy or n, n)


def need(d, x=AT, w=AT, residual=None, y=AT):
    b = ctypes.c_size_t()
    assert _lib().aep_linear_workspace_at(ctypes.byref(d), x, w, residual, y, ctypes.byref(b)) == 0
    return b.value


def plain(d):
    b = ctypes.c_size_t()
    assert _lib().aep_linear_workspace(ctypes.byref(d), ctypes.byref(b)) == 0
    return b.value


@pytest.mark.parametrize("m,n,k,fp8", [(2048, 4096, 4096, False), (2048, 4096, 4096, True), (1100, 4104, 1024, False)])
def test_room_for_copies_of_operands_that_start_off_16_bytes(m, n, k, fp8):
    d, w1 = desc(m, n, k, fp8), AT + (1 if fp8 else 2)
    base = need(d)
    xb, wb = m * k * 2, n * k * (1 if fp8 else 2)
    # (the sums of pieces, which come on top, have at most 24 M floats)
    for got, want in ((need(d, x=AT + 2), xb), (need(d, x=AT + 8), xb), (need(d, w=w1), wb), (need(d, x=AT + 2, w=w1), xb + wb)):
        assert want <= got <= want + (96 << 20), (base, got, want)
    assert base < min(xb, wb)
    assert base <= plain(d)


def test_aligned_operands_need_no_copies():
    for m, n, k in ((2048, 4096, 4096), (777, 4096, 4096), (32, 4096, 4096), (1, 14336, 4096)):
        for residual in (None, AT):
            assert need(desc(m, n, k), residual=residual) <= plain(desc(m, n, k))
        assert plain(desc(m, n, k)) == max(need(desc(m, n, k)), need(desc(m, n, k), residual=AT))


def test_products_that_gain_nothing_ask_for_nothing():
    for m, n, k in ((32, 4096, 4096), (1, 14336, 4096), (101, 1531, 1027), (0, 4096, 4096)):
        assert need(desc(m, n, k), x=AT + 2, w=AT + 2) == 0


def test_copies_have_a_bound():
    assert need(desc(64, 1 << 18, 4096), w=AT + 2) <= 96 << 20  # 2 GiB of W: not copied


def test_results_of_other_alignments_may_be_cut_otherwise():
    # what is asked for is what the call with these pointers takes: never more than it may use
    for y in (AT, AT + 2, AT + 8):
        for residual in (None, AT, AT + 2):
            assert need(desc(400, 4096, 8200), residual=residual, y=y) <= 96 << 20


def test_refusals():
    lib, b = _lib(), ctypes.c_size_t()
    d = desc(2048, 4096, 4096)
    ok = [ctypes.byref(d), AT, AT, None, AT, ctypes.byref(b)]
    assert lib.aep_linear_workspace_at(*ok) == L.AEP_OK
    for at, v in ((0, None), (1, AT + 1), (2, AT + 1), (3, AT + 1), (4, AT + 1), (5, None)):
        a = list(ok)
        a[at] = v
        assert lib.aep_linear_workspace_at(*a) == L.AEP_ERR_INVALID_ARG, at
    assert lib.aep_linear_workspace_at(ctypes.byref(desc(4, 4, 0)), AT, AT, None, AT, ctypes.byref(b)) == L.AEP_ERR_INVALID_ARG
    d.x_dtype = L.AEP_FP8_E4M3
    assert lib.aep_linear_workspace_at(*ok) == L.AEP_ERR_UNSUPPORTED
