"""CPU: heads and rows of the attention's output that overlap are refused also where their distances take more than 64
bits."""

import ctypes
import os

import pytest

from paper_2505_08944_amd import _lib as L


def status(total, heads, row, head, max_pages=1):
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libaep.so not built (run __graft_entry__.build())")
    c = L.Cache4Desc(4, 64, 1, 128)
    s = L.Cache4Seqs(16, 16, None, None, max_pages, max_pages, 1, total)
    a = L.Attend4Desc(heads, 0, 0, 1.0, 128, 128, row, head)
    return L.lib().aep_cache4_attend_workspace(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a),
                                               ctypes.byref(ctypes.c_size_t()))


def test_strides():
    most = 1 << 40
    # row r + 1 of head h is row r of head h + 1; (heads - 1) head is 2^64, or rows the same
    assert status(2, (1 << 24) + 1, most, most) == L.AEP_ERR_INVALID_ARG
    assert status((1 << 24) + 1, 2, most, most) == L.AEP_ERR_INVALID_ARG
    assert status((1 << 25) + 1, 31, most, most >> 1) == L.AEP_ERR_INVALID_ARG
    # far apart, one way and the other
    assert status(2, 1 << 20, 128, most) == L.AEP_OK
    assert status(1 << 20, 2, most, 128) == L.AEP_OK
    assert status(1 << 20, 2, most, most >> 1) == L.AEP_OK
    assert status(5, 3, 300, 100) == L.AEP_ERR_INVALID_ARG
