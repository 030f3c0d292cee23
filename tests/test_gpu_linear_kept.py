"""A Linear keeps its tensors, not copies: tensors whose shape, strides, type or device
are changed under it afterwards are refused, new values and memory are used."""

import pytest
import torch

import paper_2505_08944_amd as aep

pytestmark = pytest.mark.gpu


def kept(n=24, k=32):
    w = torch.randn(n, k, device="cuda").to(torch.bfloat16)
    b = torch.randn(n, device="cuda")
    return w, b, aep.Linear(w, bias=b, out_dtype=torch.float32), torch.randn(5, k, device="cuda").to(torch.bfloat16)


# what the tensors become: none of it is read (the call is refused on the host)
CHANGES = {
    "type": lambda w, b: setattr(w, "data", w.data.half()),
    "wider type": lambda w, b: setattr(w, "data", w.data.float()),
    "same bytes": lambda w, b: setattr(w, "data", w.data.view(torch.float16)),
    "rows": lambda w, b: setattr(w, "data", w.data[:12]),
    "columns": lambda w, b: setattr(w, "data", w.data[:, :16]),
    "transposed": lambda w, b: setattr(w, "data", w.data.t()),
    "strides": lambda w, b: setattr(w, "data", torch.zeros(24, 40, dtype=torch.bfloat16, device="cuda")[:, :32]),
    "host": lambda w, b: setattr(w, "data", w.data.cpu()),
    "bias type": lambda w, b: setattr(b, "data", b.data.to(torch.bfloat16)),
    "bias length": lambda w, b: setattr(b, "data", b.data[:12]),
    "bias strides": lambda w, b: setattr(b, "data", torch.zeros(24, 2, device="cuda")[:, 0]),
    "bias host": lambda w, b: setattr(b, "data", b.data.cpu()),
}


@pytest.mark.parametrize("what", CHANGES)
def test_changed_tensors_are_refused(what):
    w, b, lin, x = kept()
    y = lin(x)
    CHANGES[what](w, b)
    with pytest.raises(ValueError):
        lin(x)
    with pytest.raises(ValueError):
        lin(x[:2])  # a call unlike the one before
    assert y.shape == (5, 24)


def test_changed_scales_are_refused():
    w, _, _, x = kept()
    s = torch.ones(24, dtype=torch.bfloat16, device="cuda")
    lin = aep.Linear(w.to(torch.float8_e4m3fn), scale=s)
    lin(x)
    s.data = s.data.float()
    with pytest.raises(ValueError):
        lin(x)


def test_new_values_and_memory_are_used():
    w, b, lin, x = kept()
    for _ in range(2):
        w.data = torch.randn(24, 32, device="cuda").to(torch.bfloat16)
        b.data = torch.randn(24, device="cuda")
        assert torch.equal(lin(x), aep.linear(x, w, bias=b, out_dtype=torch.float32))
    w.zero_()
    assert torch.equal(lin(x), b.expand(5, 24))
