"""CPU: the memory that a layer's router reads its bias from stays the bias's, whatever
becomes of the tensor that it was given with."""

import ctypes
import os
from types import SimpleNamespace

import pytest
import torch

import paper_2505_08944_amd as aep
from paper_2505_08944_amd import _lib as L
from paper_2505_08944_amd import context


def test_the_bias_keeps_its_memory(monkeypatch):
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libaep.so not built (run __graft_entry__.build())")
    given = []

    class Lib:
        def aep_set_router(self, h, layer, desc, bias):
            given.append(bias)
            return 0

    # (host tensors, as nothing reads them)
    monkeypatch.setattr(context, "_need", lambda *a: None)
    ctx = SimpleNamespace(lib=Lib(), h=ctypes.c_void_p(), n_layers=1, n_experts=64, device=torch.device("cpu"), _bias_refs={})
    bias = torch.zeros(64)
    aep.Context.set_router(ctx, 0, aep.Router(64, 6), bias)
    assert given == [bias.data_ptr()] and ctx._bias_refs[0].data_ptr() == given[0]
    bias[3] = 1.0  # values written to the tensor are the layer's
    assert ctx._bias_refs[0][3] == 1.0
    bias.data = torch.ones(64)  # other memory is not, and the layer's own is not freed
    assert bias.data_ptr() != given[0] and ctx._bias_refs[0].data_ptr() == given[0]
    aep.Context.set_router(ctx, 0, None)
    assert given[-1] is None and ctx._bias_refs[0] is None
