"""The tiled dense product: rounds, remainder rows, cut tiles, K steps that are
not whole, against 64 bits element by element (tolerance: test_gpu_linear.py;
the activations of this kernel are off by at most 1.5e-7 |v|, which the sums'
term 1.13 (K + 16) 2^-23 S >= 2e-6 |v| covers)."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2505_08944_amd as aep
from gpu_helpers import log
from paper_2505_08944_amd import _lib as L
from test_gpu_linear import FNS, TYPES, check, f64, make

pytestmark = pytest.mark.gpu


def gpu_make(M, N, K, wdt, res, seed, pad=0):
    """As make(), drawn on the GPU; the padding is NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mat(r, c, dtype, scale):
        t = torch.full((r, c + pad), float("nan"), device="cuda")
        t[:, :c] = torch.randn(r, c, device="cuda", generator=g) * scale
        return t.to(dtype)[:, :c]

    x = mat(M, K, torch.bfloat16, 1.0)
    w = mat(N, K, TYPES[wdt], 50.0 if wdt == "fp8" else 0.5)
    s = (torch.rand(N, device="cuda", generator=g) * 0.02 + 0.001).to(torch.bfloat16) if wdt == "fp8" else None
    b = torch.randn(N, device="cuda", generator=g)
    r = mat(M, N, TYPES[res], 1.0) if res else None
    return x, w, s, b, r


def gpu_check(y, x, w, s, b, r, fn, what):
    """check() with the products on the GPU in float64."""
    xd, wd = x.double(), w.float().double()
    if s is not None:
        wd = wd * s.double()[:, None]
    v = xd @ wd.T + b.double()
    size = xd.abs() @ wd.abs().T + b.double().abs()
    F = torch.nn.functional
    a = {"none": lambda t: t, "relu": F.relu, "silu": F.silu, "gelu": F.gelu,
         "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[fn](v)
    ref = a if r is None else a + r.double()
    tol = 1.13 * (x.shape[1] + 16) * 2.0 ** -23 * size + 2.0 ** -20 * a.abs() + 2.0 ** -24 * size
    tol = tol + (2.0 ** -8 if y.dtype == torch.bfloat16 else 2.0 ** -23) * (ref.abs() + tol)
    bad = ~((y.double() - ref).abs() <= tol)
    n = int(bad.sum())
    assert n == 0, (what, n, bad.nonzero()[:4].tolist(), y[bad][:4].tolist(), ref[bad][:4].tolist())


# Products that the tile kernel takes (test_linear_plan_host.py says how each is
# cut): rows left of every height, rows of smaller tiles alone, halves and
# pieces of both, odd numbers of column halves, K steps that are not whole.
SIZES = [
    (4100, 4400, 264), (4180, 4100, 520), (4300, 4352, 1040), (8192, 2100, 1032), (4096, 4096, 328), (2500, 14000, 520),
    (777, 4096, 4096), (300, 14336, 2056), (400, 4096, 8200), (1025, 4104, 2048), (1100, 2000, 4104), (1217, 3000, 2048),
    (65, 14336, 4104), (200, 4096, 14336), (3000, 1032, 1544), (641, 2184, 4096), (2048, 4096, 2048), (1500, 6000, 1032),
    (1536, 1536, 4096), (777, 14336, 1024), (1410, 1100, 4096), (1290, 4096, 4104),
    # rows of 64-row tiles alone; the shortest K that come here
    (410, 384, 12320), (356, 4000, 2224), (22, 3160, 14912), (7823, 7536, 112),
]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("wdt", ["bf16", "fp8"])
def test_sizes(M, N, K, wdt):
    if wdt == "fp8":
        K = (K + 15) // 16 * 16
    i = SIZES.index((M, N, K)) if (M, N, K) in SIZES else len(SIZES) + K % 5
    fn, res = FNS[i % 5], [None, "bf16", "f32"][i % 3]
    log(f"tiles {M}x{N}x{K} {wdt} {fn} residual {res}")
    x, w, s, b, r = gpu_make(M, N, K, wdt, res, seed=i, pad=16 if i % 2 else 0)
    for out in (torch.bfloat16, torch.float32):
        y = aep.linear(x, w, scale=s, bias=b, activation=fn, residual=r, out_dtype=out)
        gpu_check(y, x, w, s, b, r, fn, (M, N, K, wdt, fn, out))


@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("res", [None, "bf16", "f32"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_epilogues(fn, res, out):
    x, w, s, b, r = gpu_make(1100, 4104, 1024, "bf16", res, seed=3)
    x = (x.float() * torch.linspace(0.01, 1.0, 1100, device="cuda")[:, None]).to(torch.bfloat16)
    y = aep.linear(x, w, bias=b, activation=fn, residual=r, out_dtype=TYPES[out])
    gpu_check(y, x, w, s, b, r, fn, (fn, res, out))


@pytest.mark.parametrize("M,N,K,wdt", [(400, 4096, 8200, "bf16"), (400, 4096, 8208, "fp8")])
def test_without_and_with_less_scratch(M, N, K, wdt):
    """A product that wants scratch gets none, some, or all of it."""
    x, w, s, b, r = gpu_make(M, N, K, wdt, "bf16", seed=5)
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    d = L.LinearDesc(M, N, K, L.AEP_BF16, L.AEP_FP8_E4M3 if wdt == "fp8" else L.AEP_BF16, L.AEP_BF16, L.AEP_F32,
                     L.AEP_BF16, L.AEP_FN_SILU, K, K, N, N)
    need = ctypes.c_size_t()
    lib = L.lib()
    L.check(lib.aep_linear_workspace(ctypes.byref(d), ctypes.byref(need)), "workspace")
    assert need.value > 0
    for n in (0, 1000, need.value // 2, need.value - 4, need.value):
        ws = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")
        y.fill_(0)
        L.check(lib.aep_linear(ctypes.byref(d), x.data_ptr(), w.data_ptr(), None if s is None else s.data_ptr(),
                               b.data_ptr(), r.data_ptr(), y.data_ptr(), ws.data_ptr() if n else None, n,
                               torch.cuda.current_stream().cuda_stream), "aep_linear")
        gpu_check(y, x, w, s, b, r, "silu", n)
        assert (ws[n:] == 255).all()


def test_residual_in_place_and_strides():
    M, N, K = 1100, 4104, 1032
    x, w, s, b, r = gpu_make(M, N, K, "bf16", "bf16", seed=7, pad=8)
    keep = r.clone()
    y = aep.linear(x, w, bias=b, residual=r, out=r)
    assert y is r
    gpu_check(y, x, w, s, b, keep, "none", "in place")
    for off, ld in ((0, N + 8), (1, N + 3), (4, N + 4)):
        buf = torch.full(((M + 2) * ld + off,), 77.0, dtype=torch.bfloat16, device="cuda")
        out = buf[off:off + (M + 2) * ld].view(M + 2, ld)[1:M + 1, :N]
        aep.linear(x, w, bias=b, residual=keep, out=out)
        # (rows of another alignment may take the other kernel, which adds in another order)
        gpu_check(out, x, w, s, b, keep, "none", (off, ld))
        rest = torch.ones_like(buf, dtype=torch.bool)
        rest[off:off + (M + 2) * ld].view(M + 2, ld)[1:M + 1, :N] = False
        assert (buf[rest] == 77.0).all()


def test_non_finite_values_stay_in_their_rows_and_columns():
    M, N, K = 1100, 4104, 1032
    x, w, s, b, r = gpu_make(M, N, K, "bf16", None, seed=11)
    x[7, 1031] = float("nan")
    x[1090, 0] = float("inf")
    w[333, 5] = float("-inf")
    y = aep.linear(x, w, out_dtype=torch.float32)
    ref = x.double() @ w.double().T
    assert torch.equal(y.isnan(), ref.isnan())
    assert torch.equal(y.isinf(), ref.isinf()) and torch.equal(y[y.isinf()].double(), ref[ref.isinf()])


@pytest.mark.parametrize("M,N,K,wdt", [(777, 4096, 4096, "bf16"), (4200, 4400, 256, "bf16"), (600, 4096, 4096, "fp8")])
def test_graphs_on_two_streams_and_equal_bits(M, N, K, wdt):
    x, w, s, b, r = gpu_make(M, N, K, wdt, "bf16", seed=13)
    lin = aep.Linear(w, scale=s, bias=b, activation="gelu")
    ref = lin(x, r)
    gpu_check(ref, x, w, s, b, r, "gelu", "eager")
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(lin(x, r))
        graphs.append(gr)
    torch.cuda.synchronize()
    for i in range(3):
        for o in outs:
            o.fill_(0)
        torch.cuda.synchronize()
        for gr in graphs:
            with torch.cuda.stream(torch.cuda.Stream()):
                gr.replay()
        mine = lin(x, r)
        torch.cuda.synchronize()
        assert all(torch.equal(o, ref) for o in outs) and torch.equal(mine, ref), i


@pytest.mark.parametrize("M,N,K", [(1100, 4103, 1024), (2050, 2049, 1032), (640, 4099, 4096), (1100, 4108, 1024)])
@pytest.mark.parametrize("out,res", [("bf16", None), ("bf16", "bf16"), ("bf16", "f32"), ("f32", None), ("f32", "bf16"),
                                     ("f32", "f32")])
def test_results_of_any_alignment(M, N, K, out, res):
    """Odd numbers of columns; results and residuals whose rows start anywhere; what lies around them stays."""
    x, w, s, b, _ = gpu_make(M, N, K, "bf16", None, seed=17)
    for i, (off, pad) in enumerate(((0, 0), (1, 3), (2, 2), (4, 1), (0, (-N) % 8))):
        fn = FNS[(i + N) % 5]
        log(f"tiles {M}x{N}x{K} {out} residual {res} offset {off} padding {pad} {fn}")

        def at(dtype):
            buf = torch.full((off + (M + 2) * (N + pad),), 77.0, dtype=TYPES[dtype], device="cuda")
            return buf, buf[off:].view(M + 2, N + pad)[1:M + 1, :N]

        buf, y = at(out)
        r = None
        if res:
            r = at(res)[1]
            r.copy_(torch.randn(M, N, device="cuda"))
        aep.linear(x, w, bias=b, activation=fn, residual=r, out=y, out_dtype=TYPES[out])
        gpu_check(y, x, w, s, b, r, fn, (M, N, K, out, res, off, pad))
        y.fill_(77.0)
        assert (buf == 77.0).all()


@pytest.mark.parametrize("M,N,K,wdt", [(1000, 5000, 2731, "bf16"), (777, 2003, 2001, "bf16"), (2048, 4096, 1000, "fp8"),
                                       (1000, 5000, 2731, "fp8"), (1100, 4104, 1024, "bf16"), (1100, 4104, 2048, "fp8")])
def test_operands_of_any_alignment(M, N, K, wdt):
    """Rows that start anywhere are copied into the scratch: x's, W's, or both; with too little of it the product
    runs without.  What lies between the rows (NaN) and behind the scratch is not used."""
    b = torch.randn(N, device="cuda")
    lib, need = L.lib(), ctypes.c_size_t()
    taken = 0
    for xo, xp, wo, wp in ((0, 0, 0, 0), (1, 0, 0, 0), (0, 3, 0, 0), (0, 0, 1, 0), (0, 0, 0, 5), (3, 1, 2, 7)):
        def at(r, c, off, pad, dtype, scale):
            t = torch.full((off + r * (c + pad),), float("nan"), device="cuda")
            t[off:].view(r, c + pad)[:, :c] = torch.randn(r, c, device="cuda") * scale
            return t.to(dtype)[off:].view(r, c + pad)[:, :c]

        x = at(M, K, xo, xp, torch.bfloat16, 1.0)
        w = at(N, K, wo, wp, TYPES[wdt], 50.0 if wdt == "fp8" else 0.5)
        s = (torch.rand(N, device="cuda") * 0.02 + 0.001).to(torch.bfloat16) if wdt == "fp8" else None
        log(f"operands {M}x{N}x{K} {wdt} offsets {xo} {wo} padding {xp} {wp}")
        y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        d = L.LinearDesc(M, N, K, L.AEP_BF16, L.AEP_FP8_E4M3 if wdt == "fp8" else L.AEP_BF16, L.AEP_BF16, L.AEP_F32,
                         L.AEP_BF16, L.AEP_FN_GELU, K + xp, K + wp, N, N)
        L.check(lib.aep_linear_workspace(ctypes.byref(d), ctypes.byref(need)), "workspace")
        full = M * (K + 16) * 2 + N * (K + 16) * 2 + need.value  # enough for copies of misaligned pointers as well
        for n in (0, need.value, need.value // 2, full // 16 * 16):
            ws = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")
            y.fill_(0)
            L.check(lib.aep_linear(ctypes.byref(d), x.data_ptr(), w.data_ptr(), None if s is None else s.data_ptr(),
                                   b.data_ptr(), None, y.data_ptr(), ws.data_ptr() if n else None, n,
                                   torch.cuda.current_stream().cuda_stream), "aep_linear")
            gpu_check(y, x, w, s, b, None, "gelu", (M, N, K, wdt, xo, xp, wo, wp, n))
            assert (ws[n:] == 255).all()
            taken += int(n > 0 and not bool((ws[:n] == 255).all()))
        lin = aep.linear(x, w, scale=s, bias=b, activation="gelu")
        gpu_check(lin, x, w, s, b, None, "gelu", (M, N, K, wdt, xo, xp, wo, wp, "binding"))
    assert taken  # copies were made


def test_copied_operands_in_graphs():
    x, w, s, b, r = gpu_make(1000, 5000, 2731, "bf16", "bf16", seed=21)
    lin = aep.Linear(w, bias=b, activation="silu")
    ref = lin(x, r)
    gpu_check(ref, x, w, s, b, r, "silu", "eager")
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(lin(x, r))
        graphs.append(gr)
    torch.cuda.synchronize()
    for i in range(3):
        for o in outs:
            o.fill_(0)
        torch.cuda.synchronize()
        for gr in graphs:
            with torch.cuda.stream(torch.cuda.Stream()):
                gr.replay()
        mine = lin(x, r)
        torch.cuda.synchronize()
        assert all(torch.equal(o, ref) for o in outs) and torch.equal(mine, ref), i
