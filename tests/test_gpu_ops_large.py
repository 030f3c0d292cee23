"""The dense product and routing at sizes whose launches have more than 2^32
threads, or that 32-bit arguments cannot hold; what is kept between calls."""

import pytest
import torch

import paper_2505_08944_amd as aep
from gpu_helpers import log

pytestmark = pytest.mark.gpu


def test_rows_up_to_the_limit():
    m = 1 << 30
    log(f"linear {m}x1x1")
    x = torch.ones(m, 1, dtype=torch.bfloat16, device="cuda")
    x[::65537] = 3.0
    w = torch.full((1, 1), 0.5, dtype=torch.bfloat16, device="cuda")
    y = aep.linear(x, w)
    assert torch.equal(y, x.mul_(0.5))  # exact
    del x, y
    log("more rows than that")
    x = torch.empty(m + 1, 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(aep.AEPError):
        aep.linear(x, w)
    with pytest.raises(aep.AEPError):
        aep.linear(w, x)


@pytest.mark.parametrize("E,T", [(2, (1 << 28) + 5), (300, (1 << 24) + 3)])
def test_many_tokens(E, T):
    log(f"route {T} tokens, {E} experts")
    logits = torch.zeros(T, E, device="cuda")
    want = torch.arange(T, device="cuda", dtype=torch.int32).mul_(7).remainder_(E)
    step = 1 << 24
    for a in range(0, T, step):
        logits[a:a + step].scatter_(1, want[a:a + step].long()[:, None], 1.0)
    idx, w = aep.route(aep.Router(E, 1), logits)
    assert torch.equal(idx.view(-1), want)
    assert (w == 1.0).all()


def test_attributes_are_fixed():
    w = torch.ones(8, 16, dtype=torch.bfloat16, device="cuda")
    lin, r = aep.Linear(w), aep.Router(8, 2)
    for o, name, v in ((lin, "weight", w[:4]), (lin, "k", 8), (lin, "out_dtype", torch.float32), (r, "top_k", 4),
                       (r, "n_experts", 4)):
        with pytest.raises(AttributeError):
            setattr(o, name, v)
    x = torch.ones(3, 16, dtype=torch.bfloat16, device="cuda")
    assert (lin(x) == 16).all()
    w.fill_(2.0)  # its values are the tensor's
    assert (lin(x) == 32).all()
