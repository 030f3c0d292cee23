"""The activations' own errors, by value (aep.h): x is zero, so the sum is exactly the
f32 bias, which holds the activation's arguments; for each kernel of the product.

f32 results: 2^-20 of their value and 2^-142.  bf16: 2^-15 of it before the
rounding of 2^-8, GELU 2^-23 |v| more, and 2^-119 (bf16 has steps of 2^-133 down
there).  A residual adds half a step of the result, 2^-24 or 2^-8."""

import numpy as np
import pytest
import torch

import paper_2505_08944_amd as aep
from gpu_helpers import log
from test_linear_fn_host import FNS, reference

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# (M, N, K, type of x and W): the row kernel; the tile kernel: whole tiles, column halves,
# pieces along K, 128- and 64-row tiles (test_linear_plan_host.py's sizes)
SIZES = [(4, 2000, 64, "bf16"), (40, 2003, 64, "f32"), (2048, 4096, 2048, "bf16"), (4096, 4096, 328, "bf16"),
         (777, 4096, 4096, "bf16"), (400, 4096, 8200, "bf16"), (410, 384, 12320, "bf16"), (1100, 4103, 1024, "bf16"),
         (2048, 4096, 2048, "fp8")]


def arguments(N, seed):
    g = np.random.default_rng(seed)
    v = np.concatenate([np.linspace(-108, 20, N // 2), np.linspace(-9, 6, N - N // 2 - N // 8), g.standard_normal(N // 8)])
    g.shuffle(v)
    v[:6] = [0.0, -0.0, 1e30, -1e30, -88.8, 2.0 ** -140]
    return torch.from_numpy(v.astype(np.float32))


@pytest.mark.parametrize("M,N,K,t", SIZES)
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
def test_activations_by_value(M, N, K, t, out, residual):
    if t == "f32" and out == "bf16":
        pytest.skip("f32 products have f32 results")
    log(f"activations {M}x{N}x{K} {t} {out} residual {residual}")
    b = arguments(N, M)
    x = torch.zeros(M, K, dtype=TYPES.get(t, torch.bfloat16), device="cuda")
    w = torch.ones(N, K, device="cuda").to(torch.float8_e4m3fn if t == "fp8" else x.dtype)
    scale = torch.ones(N, dtype=torch.bfloat16, device="cuda") if t == "fp8" else None
    r = torch.full((M, N), -0.25, dtype=TYPES[out], device="cuda") if residual else None
    for fn in FNS:
        y = aep.linear(x, w, scale=scale, bias=b.cuda(), activation=fn, residual=r, out_dtype=TYPES[out])
        assert bool((y == y[0]).all()), fn  # every row alike
        v = b.double().numpy()
        act = reference(fn, v)
        if out == "f32":
            tol = 2.0 ** -20 * np.abs(act) + 2.0 ** -142
        else:
            tol = 2.0 ** -15 * np.abs(act) + (2.0 ** -23 * np.abs(v) if fn == "gelu" else 0.0) + 2.0 ** -119
        ref = act - 0.25 if residual else act
        tol = tol + (2.0 ** -8 * (np.abs(ref) + tol) + 2.0 ** -134 if out == "bf16" else 2.0 ** -24 * np.abs(ref) if residual else 0.0)
        got = y[0].double().cpu().numpy()
        bad = ~(np.abs(got - ref) <= tol)
        assert not bad.any(), (fn, int(bad.sum()), v[bad][:4], got[bad][:4], ref[bad][:4])


@pytest.mark.parametrize("M", [3, 2048])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_values_that_are_not_finite(M, out):
    N = 4096
    x, w = torch.zeros(M, 2048, dtype=torch.bfloat16, device="cuda"), torch.ones(N, 2048, dtype=torch.bfloat16, device="cuda")
    b = torch.zeros(N, device="cuda")
    b[5], b[6], b[700] = float("nan"), float("inf"), float("-inf")
    for fn in FNS:
        y = aep.linear(x, w, bias=b, activation=fn, out_dtype=TYPES[out])
        assert y[:, 5].isnan().all() and (y[:, 6] == float("inf")).all()
        assert (y[:, 700] == (0.0 if fn == "relu" else float("-inf"))).all() if fn in ("relu", "none") else \
            not y[:, 700].isinf().any()
        y[:, [5, 6, 700]] = 0.0
        assert not y.any()
