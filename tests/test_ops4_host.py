"""CPU checks of the calls on 4-bit data: what they refuse, before anything is launched."""

import ctypes
import os

import pytest

from paper_2505_08944_amd import _lib as L

INVALID, UNSUPPORTED = L.AEP_ERR_INVALID_ARG, L.AEP_ERR_UNSUPPORTED


def _lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libaep.so not built (run __graft_entry__.build())")
    return L.lib()


def test_quantiser():
    lib = _lib()
    #     x, type, ld, rows, k, codes, scale, stream
    ok = [16, 1, 40, 4, 40, 16, 16, None]
    for at, v, st in ((0, None, 1), (0, 17, 1), (1, 3, 1), (1, -1, 1), (1, 2, 6), (2, 39, 1), (3, -1, 1), (4, 0, 1),
                      (5, None, 1), (6, None, 1), (3, 1 << 39, 6)):
        a = list(ok)
        a[at] = v
        assert lib.aep_mx4_quantize(*a) == st, (at, v)
        # codes, scale, rows, k, y, type, ld, stream
        assert lib.aep_mx4_dequantize(a[5], a[6], a[3], a[4], a[0], a[1], a[2], None) == st, (at, v)
    assert lib.aep_mx4_quantize(18, 0, 40, 4, 40, 16, 16, None) == INVALID  # f32 at 2 bytes
    assert lib.aep_mx4_quantize(16, 0, (1 << 30) + 1, 4, (1 << 30) + 1, 16, 16, None) == UNSUPPORTED
    assert lib.aep_mx4_quantize(None, 0, 40, 0, 40, None, None, None) == L.AEP_OK


def test_more_blocks_than_are_counted():
    """2^38 blocks at most, also where rows times blocks of a row are more than 64 bits hold."""
    lib = _lib()
    for rows, k in ((1 << 38, 1 << 30), ((1 << 38) - 1, 1 << 30), ((1 << 13) + 1, 1 << 30), (1 << 38, 33), ((1 << 38) + 1, 1)):
        assert lib.aep_mx4_quantize(16, 0, 1 << 30, rows, k, 16, 16, None) == UNSUPPORTED
        assert lib.aep_mx4_dequantize(16, 16, rows, k, 16, 0, 1 << 30, None) == UNSUPPORTED


def test_weights():
    lib = _lib()
    n = ctypes.c_size_t()
    assert lib.aep_linear4_packed_bytes(17, 129, ctypes.byref(n)) == 0 and n.value == 2 * 2 * 1088
    assert lib.aep_linear4_packed_bytes(17, 129, None) == INVALID
    for a, b, st in ((0, 4, 1), (4, 0, 1), (-1, 4, 1), ((1 << 30) + 1, 4, 6), (4, (1 << 30) + 1, 6), (1 << 30, 1 << 11, 6)):
        assert lib.aep_linear4_packed_bytes(a, b, ctypes.byref(n)) == st
        assert lib.aep_linear4_pack(16, 16, a, b, 16, None) == st
    for args in ((None, 16, 16), (16, None, 16), (16, 16, None), (16, 16, 24)):
        assert lib.aep_linear4_pack(args[0], args[1], 4, 4, args[2], None) == INVALID


def _linear(**kw):
    a = dict(m=4, n=16, k=32, y_dtype=1, bias_dtype=0, res_dtype=1, fn=0, ldx=32, ldy=16, ldr=16)
    a.update(kw)
    return L.Linear4Desc(**a)


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), 1), (dict(n=0), 1), (dict(k=0), 1), (dict(ldx=31), 1), (dict(ldy=15), 1), (dict(fn=5), 1), (dict(fn=-1), 1),
    (dict(y_dtype=3), 1), (dict(bias_dtype=-1), 1), (dict(res_dtype=9), 1), (dict(y_dtype=2), 6), (dict(bias_dtype=2), 6),
    (dict(res_dtype=2), 6), (dict(m=(1 << 30) + 1), 6), (dict(m=1 << 20, n=(1 << 18) + 1, ldy=1 << 20, ldr=1 << 20), 6)])
def test_linear4_descriptions(kw, status):
    lib = _lib()
    l, n = ctypes.byref(_linear(**kw)), ctypes.c_size_t()
    assert lib.aep_linear4(l, 16, 16, None, None, 16, None, 0, None) == status
    assert lib.aep_linear4_workspace(l, 16, None, 16, ctypes.byref(n)) == status


def test_linear4_arguments():
    lib = _lib()
    d = _linear()
    ok = [ctypes.byref(d), 1024, 2048, None, None, 4096, None, 0, None]
    #        no description, x, w, y; misaligned x, w, bias (f32), residual, y, scratch
    for at, v in ((0, None), (1, None), (2, None), (5, None), (1, 1025), (2, 2056), (3, 18), (4, 4097), (5, 4097), (6, 24)):
        a = list(ok)
        a[at] = v
        assert lib.aep_linear4(*a) == INVALID, (at, v)
    for kw in (dict(res_dtype=0), dict(ldr=20), dict(ldr=15)):
        assert lib.aep_linear4(ctypes.byref(_linear(**kw)), 1024, 2048, None, 4096, 4096, None, 0, None) == INVALID
    assert lib.aep_linear4(ctypes.byref(_linear(m=0)), None, None, None, None, None, None, 0, None) == L.AEP_OK
    assert lib.aep_linear4_workspace(ctypes.byref(d), 16, None, 16, None) == INVALID


def test_linear4_scratch():
    """Few rows need none; many have the widened weights in it, and x where its rows are not aligned."""
    lib, n = _lib(), ctypes.c_size_t()

    def need(m, n_, k, x=16, **kw):
        assert lib.aep_linear4_workspace(ctypes.byref(_linear(m=m, n=n_, k=k, ldx=k, ldy=n_, ldr=n_, **kw)), x, None, 16,
                                         ctypes.byref(n)) == 0
        return n.value

    assert need(1, 14336, 4096) == 0 and need(32, 4096, 4096) == 0 and need(0, 4096, 4096) == 0
    wide = 2 * 4096 * 4096
    assert wide <= need(2048, 4096, 4096) < wide + (100 << 20)
    assert need(2048, 4096, 4096, x=18) >= wide + 2 * 2048 * 4096
    assert need(2048, 4096, 4093) >= wide + 2 * 2048 * 4096


def _cache(**kw):
    a = dict(n_pages=4, page_size=64, n_heads=2, head_dim=128)
    a.update(kw)
    return L.Cache4Desc(**a)


def _seqs(**kw):
    a = dict(pages=16, lens=16, rows=None, flag=None, ld_pages=2, max_pages=2, batch=3, total=6)
    a.update(kw)
    return L.Cache4Seqs(**a)


def _desc(**kw):
    a = dict(n_heads=8, window=0, max_rows=0, scale=1.0, q_row=1024, q_head=128, out_row=1024, out_head=128)
    a.update(kw)
    return L.Attend4Desc(**a)


def _calls(c=None, s=None, a=None, mem=256, k=256, v=256, ws=256, size=1 << 40, lse=None):
    """Statuses of append, read and attend."""
    lib = L.lib()
    c, s, a = (ctypes.byref(t) if t is not None else None for t in (c, s, a))
    return [lib.aep_cache4_append(c, mem, s, k, 256, 128, v, 256, 128, None), lib.aep_cache4_read(c, mem, s, k, v, None),
            lib.aep_cache4_attend(c, mem, s, a, k, v, lse, ws, size, None)]


@pytest.mark.parametrize("kw,status", [
    (dict(n_pages=0), 1), (dict(n_heads=0), 1), (dict(page_size=0), 1), (dict(head_dim=0), 1), (dict(page_size=16), 6),
    (dict(page_size=48), 6), (dict(page_size=8192), 6), (dict(head_dim=96), 6), (dict(head_dim=512), 6),
    (dict(n_heads=1025), 6), (dict(n_pages=1 << 30, page_size=4096), 6)])
def test_caches(kw, status):
    lib, n = _lib(), ctypes.c_size_t()
    assert lib.aep_cache4_bytes(ctypes.byref(_cache(**kw)), ctypes.byref(n)) == status
    assert _calls(_cache(**kw), _seqs(), _desc(n_heads=1025 * 8 if kw.get("n_heads", 2) == 1025 else 8)) == [status] * 3


def test_cache_bytes():
    lib, n = _lib(), ctypes.c_size_t()
    assert lib.aep_cache4_bytes(ctypes.byref(_cache()), ctypes.byref(n)) == 0
    assert n.value == 2 * 4 * 64 * 2 * (128 // 2 + 128 // 32)
    assert lib.aep_cache4_bytes(ctypes.byref(_cache()), None) == INVALID
    assert lib.aep_cache4_bytes(None, ctypes.byref(n)) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), 1), (dict(total=-1), 1), (dict(max_pages=-1), 1), (dict(ld_pages=1), 1), (dict(total=7), 1),
    (dict(pages=None), 1), (dict(lens=None), 1), (dict(pages=18), 1), (dict(lens=18), 1), (dict(rows=18), 1), (dict(flag=18), 1),
    (dict(batch=0), 1), (dict(total=(1 << 30) + 2), 6), (dict(batch=(1 << 24) + 1, rows=16), 6),
    (dict(max_pages=(1 << 24) + 1, ld_pages=1 << 25), 6)])
def test_sequences(kw, status):
    _lib()
    assert _calls(_cache(), _seqs(**kw), _desc()) == [status] * 3


@pytest.mark.parametrize("kw,status", [
    (dict(n_heads=0), 1), (dict(n_heads=7), 1), (dict(window=-1), 1), (dict(max_rows=-1), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(scale=3e38), 1), (dict(q_row=-1), 1), (dict(q_head=-1), 1), (dict(out_row=-1), 1),
    (dict(out_head=-1), 1), (dict(out_head=127), 1), (dict(out_row=1023), 1), (dict(out_row=0), 1), (dict(q_row=1 << 41), 6),
    (dict(out_row=1 << 41), 6)])
def test_attention_descriptions(kw, status):
    lib, n = _lib(), ctypes.c_size_t()
    assert _calls(_cache(), _seqs(), _desc(**kw))[2] == status
    assert lib.aep_cache4_attend_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs()), ctypes.byref(_desc(**kw)),
                                           ctypes.byref(n)) == status


def test_arguments():
    lib, n = _lib(), ctypes.c_size_t()
    assert _calls(None, _seqs(), _desc()) == [INVALID] * 3
    assert _calls(_cache(), None, _desc()) == [INVALID] * 3
    assert _calls(_cache(), _seqs(), None)[2] == INVALID
    for kw in (dict(mem=None), dict(mem=264), dict(k=None), dict(v=None), dict(k=257), dict(v=257)):
        assert _calls(_cache(), _seqs(), _desc(), **kw) == [INVALID] * 3, kw
    assert _calls(_cache(), _seqs(), _desc(), lse=18)[2] == INVALID
    assert _calls(_cache(), _seqs(), _desc(), ws=264)[2] == INVALID
    assert lib.aep_cache4_attend_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs()), ctypes.byref(_desc()),
                                           ctypes.byref(n)) == 0
    assert n.value > 0
    assert _calls(_cache(), _seqs(), _desc(), size=n.value - 1)[2] == L.AEP_ERR_CAPACITY
    assert _calls(_cache(), _seqs(), _desc(), ws=None)[2] == L.AEP_ERR_CAPACITY
    # more units than 31 bits count
    s = _seqs(total=1 << 20, batch=1 << 10, max_pages=1 << 14, ld_pages=1 << 14)
    assert _calls(_cache(), s, _desc(n_heads=1024, q_row=1 << 17, out_row=1 << 17))[2] == UNSUPPORTED
    # heads in front of rows
    d = _desc(out_row=128, out_head=128 * 6)
    assert lib.aep_cache4_attend_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs()), ctypes.byref(d), ctypes.byref(n)) == 0
    d = _desc(out_row=128, out_head=128 * 5)
    assert lib.aep_cache4_attend_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs()), ctypes.byref(d),
                                           ctypes.byref(n)) == INVALID
    # nothing to do
    assert _calls(_cache(), _seqs(total=0), _desc(), mem=None, k=None, v=None, ws=None, size=0) == [L.AEP_OK] * 3
    assert _calls(_cache(), _seqs(total=6, batch=0, rows=16), _desc(), mem=None, ws=None) == [L.AEP_OK] * 3


def test_calls_refuse_what_is_no_device_tensor():
    import numpy as np
    import torch

    import paper_2505_08944_amd as aep
    _lib()
    codes, scale = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)
    for bad in (np.zeros((4, 8), np.float32), None, [[0.0] * 8], torch.zeros(4, 8)):
        with pytest.raises(ValueError):
            aep.quantize_mx4(bad)
        with pytest.raises(ValueError):
            aep.dequantize_mx4(bad, scale, 32)
        with pytest.raises(ValueError):
            aep.Linear4(bad, scale)
    with pytest.raises(ValueError):
        aep.Cache4(4, 2, 64, device="cpu")
    for args in ((0, 2, 64), (4, 2, 80)):
        with pytest.raises(L.AEPError):
            aep.Cache4(*args, device="cpu")
