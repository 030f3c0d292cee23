"""CPU: numbers that the library's 32-bit arguments cannot hold are refused by the
binding (ctypes would cut them off), as are those that are no whole numbers."""

import os
from types import SimpleNamespace

import pytest
import torch

import paper_2505_08944_amd as aep
from paper_2505_08944_amd import _lib as L

GOOD = dict(n_experts=64, top_k=6, n_groups=8, top_groups=3, group_top=1)


def _lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libaep.so not built (run __graft_entry__.build())")
    return L.lib()


@pytest.mark.parametrize("name", sorted(GOOD))
@pytest.mark.parametrize("off", [1 << 32, -(1 << 32), 1 << 33, 1 << 64])
def test_router_refuses_what_32_bits_cut_off(name, off):
    _lib()
    aep.Router(**GOOD)
    with pytest.raises(aep.AEPError):
        aep.Router(**dict(GOOD, **{name: GOOD[name] + off}))


@pytest.mark.parametrize("name", sorted(GOOD))
def test_router_refuses_fractions(name):
    _lib()
    with pytest.raises((TypeError, ValueError)):
        aep.Router(**dict(GOOD, **{name: GOOD[name] + 0.0}))


@pytest.mark.parametrize("layer", [-1, 2, 1 << 32, (1 << 32) + 1, -(1 << 32)])
def test_set_router_refuses_layers_that_are_not_there(layer):
    """(A context without a GPU: its host state is enough.)"""
    import ctypes
    lib = _lib()
    cfg = L.Config(2, 64, 0, 64, 64, 6, 1, L.AEP_BF16, L.AEP_BF16, 16, 0)
    h = ctypes.c_void_p()
    assert lib.aep_create(ctypes.byref(cfg), ctypes.byref(h)) == 0
    try:
        ctx = SimpleNamespace(lib=lib, h=h, n_layers=2, n_experts=64, device=torch.device("cpu"), _bias_refs={})
        with pytest.raises(aep.AEPError):
            aep.Context.set_router(ctx, layer, aep.Router(**GOOD))
        assert not ctx._bias_refs
        aep.Context.set_router(ctx, 1, aep.Router(**GOOD))
    finally:
        lib.aep_destroy(h)
