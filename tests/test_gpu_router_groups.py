"""Routing by scores: groups compared by their logits where the whole selection
is redone in 64 bits (more chosen experts in one lane than it keeps at hand).

Ids equal those of the 64-bit form (ops_ref.route), weights as in test_gpu_router.py."""

import pytest
import torch

import paper_2505_08944_amd as aep
from gpu_helpers import log
from test_gpu_router import check, rule

pytestmark = pytest.mark.gpu

# no bias and group_top 1: a group is worth its largest logit.  k above the eight
# experts that a lane keeps at hand, E above the 8 per lane that it can list whole.
BY_LOGIT = [
    dict(E=256, k=16, n_groups=16, top_groups=1), dict(E=256, k=12, n_groups=16, top_groups=2),
    dict(E=160, k=10, n_groups=16, top_groups=3), dict(E=512, k=16, n_groups=32, top_groups=2),
    dict(E=480, k=9, n_groups=16, top_groups=2), dict(E=240, k=12, n_groups=3, top_groups=2),
    dict(E=510, k=14, n_groups=3, top_groups=2),
]


def crowded(c, T, seed, scale, shift):
    """Logits whose largest lie in one lane's experts: a run of E / lanes, and every 16th or 32nd."""
    g = torch.Generator().manual_seed(seed)
    E, lanes = c["E"], 16 if c["E"] <= 256 else 32
    l = torch.randn(T, E, generator=g)
    if lanes % c["n_groups"]:  # experts lane, lane + lanes, ... are one lane's
        l[torch.arange(T)[:, None], (torch.arange(T) % lanes)[:, None] + torch.arange(0, E - lanes + 1, lanes)[None]] += 3.0
    return l * scale + shift


@pytest.mark.parametrize("c", BY_LOGIT, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
# scores all alike: 1 in 64 bits above 37, 0 of a softmax 745 below the largest logit
@pytest.mark.parametrize("scale,shift", [(1.0, 0.0), (2.0, 60.0), (1000.0, 0.0)])
def test_groups_by_logits(c, score, scale, shift):
    c = dict(c, score=score)
    log(f"groups by logits {c} scale {scale} shift {shift}")
    r = aep.Router(c["E"], c["k"], **rule(c))
    for T in (1, 70):
        l = crowded(c, T, 7 * T, scale, shift)
        idx, w = aep.route(r, l.cuda())
        check(c, l, None, idx, w)
