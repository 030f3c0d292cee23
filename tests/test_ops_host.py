"""CPU checks of the calls that need no context, and of aep_set_router: what
they refuse, before anything is launched."""

import ctypes

import pytest

from paper_2505_08944_amd import _lib as L
import os


def _lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libaep.so not built (run __graft_entry__.build())")
    return L.lib()


def _router(**kw):
    a = dict(n_experts=64, top_k=6, score=0, n_groups=8, top_groups=3, group_top=1, renorm=1, scale=1.0)
    a.update(kw)
    return L.RouterDesc(**a)


BAD_ROUTERS = [
    (dict(n_experts=0), 1), (dict(top_k=0), 1), (dict(top_k=65, n_groups=1, top_groups=1), 1), (dict(score=2), 1),
    (dict(score=-1), 1), (dict(n_groups=0), 1), (dict(n_groups=7), 1), (dict(n_groups=128, n_experts=256), 1),
    (dict(top_groups=0), 1), (dict(top_groups=9), 1), (dict(top_groups=1, top_k=9), 1), (dict(group_top=0), 1),
    (dict(group_top=3), 1), (dict(renorm=2), 1), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(scale=-1.0), 1), (dict(n_experts=520), 6),
    (dict(top_k=17), 6),
]


@pytest.mark.parametrize("kw,status", BAD_ROUTERS)
def test_route_refuses_routers(kw, status):
    lib = _lib()
    r = _router(**kw)
    ld = max(1, r.n_experts)
    assert lib.aep_route_topk(ctypes.byref(r), 16, ld, None, 4, 16, 16, None, None) == status
    assert lib.aep_route_topk(ctypes.byref(r), None, ld, None, 0, None, None, None, None) == status


def test_route_refuses_arguments():
    lib = _lib()
    r = ctypes.byref(_router())
    ok = [r, 16, 64, None, 4, 16, 16, None, None]
    for at, v in ((0, None), (1, None), (1, 18), (2, 63), (3, 2), (4, -1), (5, None), (5, 1), (6, None), (6, 2), (7, 2)):
        a = list(ok)
        a[at] = v
        assert lib.aep_route_topk(*a) == L.AEP_ERR_INVALID_ARG, (at, v)
    assert lib.aep_route_topk(r, None, 64, None, 0, None, None, None, None) == L.AEP_OK


def test_set_router():
    lib = _lib()
    cfg = L.Config(2, 64, 0, 64, 64, 6, 1, L.AEP_BF16, L.AEP_BF16, 16, 0)
    h = ctypes.c_void_p()
    assert lib.aep_create(ctypes.byref(cfg), ctypes.byref(h)) == 0
    try:
        r = _router()
        assert lib.aep_set_router(h, 1, ctypes.byref(r), None) == 0
        assert lib.aep_set_router(h, 1, None, None) == 0
        assert lib.aep_set_router(None, 1, ctypes.byref(r), None) == 1
        assert lib.aep_set_router(h, 2, ctypes.byref(r), None) == 1
        assert lib.aep_set_router(h, -1, ctypes.byref(r), None) == 1
        assert lib.aep_set_router(h, 0, None, 16) == 1       # a bias without a router
        assert lib.aep_set_router(h, 0, ctypes.byref(r), 18) == 1
        for kw in (dict(n_experts=32), dict(top_k=5)):       # not the context's
            assert lib.aep_set_router(h, 0, ctypes.byref(_router(**kw)), None) == 1
        for kw, status in BAD_ROUTERS:
            assert lib.aep_set_router(h, 0, ctypes.byref(_router(**kw)), None) == status
    finally:
        lib.aep_destroy(h)


def _linear(**kw):
    a = dict(m=4, n=16, k=32, x_dtype=1, w_dtype=1, y_dtype=1, bias_dtype=0, res_dtype=1, fn=0, ldx=32, ldw=32, ldy=16,
             ldr=16)
    a.update(kw)
    return L.LinearDesc(**a)


BAD_LINEARS = [
    (dict(m=-1), 1), (dict(n=0), 1), (dict(k=0), 1), (dict(ldx=31), 1), (dict(ldw=31), 1), (dict(ldy=15), 1),
    (dict(fn=5), 1), (dict(fn=-1), 1), (dict(x_dtype=3), 1), (dict(w_dtype=-1), 1), (dict(y_dtype=9), 1),
    (dict(bias_dtype=4), 1), (dict(res_dtype=-2), 1), (dict(x_dtype=2), 6), (dict(w_dtype=0), 6),
    (dict(x_dtype=0), 6), (dict(x_dtype=0, w_dtype=0), 6), (dict(y_dtype=2), 6), (dict(bias_dtype=2), 6),
    (dict(res_dtype=2), 6), (dict(m=(1 << 30) + 1), 6), (dict(k=(1 << 30) + 1, ldx=1 << 31, ldw=1 << 31), 6),
    (dict(m=1 << 20, n=(1 << 18) + 1, ldy=1 << 20, ldr=1 << 20), 6),
]


@pytest.mark.parametrize("kw,status", BAD_LINEARS)
def test_linear_refuses_descriptions(kw, status):
    lib = _lib()
    l = ctypes.byref(_linear(**kw))
    n = ctypes.c_size_t()
    assert lib.aep_linear(l, 16, 16, None, None, None, 16, None, 0, None) == status
    assert lib.aep_linear_workspace(l, ctypes.byref(n)) == status


def test_linear_refuses_arguments():
    lib = _lib()
    d = _linear()
    ok = [ctypes.byref(d), 1024, 2048, None, None, None, 4096, None, 0, None]
    #        no x, w, y; a scale without fp8; misaligned x, w, bias (f32), residual, y, scratch
    for at, v in ((0, None), (1, None), (2, None), (6, None), (3, 16), (1, 1025), (2, 2049), (4, 18), (5, 4097),
                  (6, 4097), (7, 24)):
        a = list(ok)
        a[at] = v
        assert lib.aep_linear(*a) == L.AEP_ERR_INVALID_ARG, (at, v)
    fp8 = ctypes.byref(_linear(w_dtype=2))
    assert lib.aep_linear(fp8, 1024, 2048, None, None, None, 4096, None, 0, None) == L.AEP_ERR_INVALID_ARG
    assert lib.aep_linear(fp8, 1024, 2048, 17, None, None, 4096, None, 0, None) == L.AEP_ERR_INVALID_ARG
    # the residual in y's place, in another type, stride, or with short rows
    for kw in (dict(res_dtype=0), dict(ldr=20), dict(ldr=15)):
        assert lib.aep_linear(ctypes.byref(_linear(**kw)), 1024, 2048, None, None, 4096, 4096, None, 0,
                              None) == L.AEP_ERR_INVALID_ARG
    # no rows: nothing to do
    assert lib.aep_linear(ctypes.byref(_linear(m=0)), None, None, None, None, None, None, None, 0, None) == L.AEP_OK
    assert lib.aep_linear_workspace(ctypes.byref(d), None) == L.AEP_ERR_INVALID_ARG


def test_calls_refuse_what_is_no_device_tensor():
    import numpy as np
    import torch

    import paper_2505_08944_amd as aep
    _lib()
    r = aep.Router(8, 2)
    for bad in (np.zeros((4, 8), np.float32), None, [[0.0] * 8], torch.zeros(4, 8)):
        with pytest.raises(ValueError):
            aep.route(r, bad)
        with pytest.raises(ValueError):
            aep.Linear(bad)
