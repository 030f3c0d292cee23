"""aep_linear against a 64-bit product, element by element.

Tolerance.  The f32 sum of K exact products (of 64-bit size sum S of their
absolute values) and a bias is off by at most (K + 16) 2^-23 S in any order,
whether a step rounds (2^-24 of what has been added up, at most S) or cuts
off (2^-23).  An fp8 scale multiplies it: 2^-24.  The activations' slopes are
at most 1.13, their own error at most 2^-20 of their value for bf16 results
and 2^-21 for f32 ones; GELU's erfc argument is off by 2^-23 relative, which
changes erfc by at most |z| * 2 / sqrt(pi) e^(-z^2) * 2^-23 <= 2^-23, times
|v| / 2.  Adding the residual and rounding: half a step of the result each,
2^-24 (f32) or 2^-8 (bf16).
"""

import numpy as np
import pytest
import torch

import ops_ref
import paper_2505_08944_amd as aep
from gpu_helpers import log

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
FNS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def make(M, N, K, wdt="bf16", bias="f32", res="bf16", seed=0, pad=0, off=0):
    """Device tensors; pad: unused elements after each row (NaN), off: elements before the first."""
    g = torch.Generator().manual_seed(seed)
    act = torch.float32 if wdt == "f32" else torch.bfloat16

    def mat(r, c, dtype, scale=1.0):
        t = torch.full((off + r * (c + pad),), float("nan"), dtype=torch.float32)
        v = t[off:].view(r, c + pad)[:, :c]
        v.copy_(torch.randn(r, c, generator=g) * scale)
        if dtype == torch.float8_e4m3fn:
            t = (t * 100).clamp(-448, 448)
        return t.to(dtype).cuda()[off:].view(r, c + pad)[:, :c]

    x, w = mat(M, K, act), mat(N, K, TYPES[wdt], 0.5)
    scale = (torch.rand(N, generator=g) * 0.02 + 0.001).to(torch.bfloat16).cuda() if wdt == "fp8" else None
    b = (torch.randn(N, generator=g)).to(TYPES[bias]).cuda() if bias else None
    r = mat(M, N, TYPES[res]) if res else None
    return x, w, scale, b, r


def f64(t):
    return None if t is None else t.float().cpu().numpy().astype(np.float64)


def check(y, x, w, scale, b, r, fn, what):
    with np.errstate(invalid="ignore"):
        ref, size = ops_ref.linear(f64(x), f64(w), f64(scale), f64(b), fn, f64(r))
    K = x.shape[1]
    v = ref if r is None else ref - f64(r)
    tol = 1.13 * (K + 16) * 2.0 ** -23 * size + 2.0 ** -20 * np.abs(v) + 2.0 ** -24 * size
    if fn == "gelu":
        tol = tol + 2.0 ** -24 * size
    tol = tol + (2.0 ** -8 if y.dtype == torch.bfloat16 else 2.0 ** -23) * (np.abs(ref) + tol)
    got = f64(y)
    err = np.abs(got - ref)
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], tol[bad][:4])


SIZES = [
    (1, 1, 1), (1, 1, 8), (1, 16, 64), (2, 7, 16), (1, 130, 512), (16, 16, 64), (17, 65, 72), (15, 64, 2048),
    (32, 64, 128), (33, 48, 1000), (48, 100, 65), (64, 256, 320), (65, 129, 96), (100, 300, 1027), (130, 70, 63),
    (200, 257, 520), (257, 513, 192), (300, 40, 1500),
]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("wdt", ["bf16", "fp8", "f32"])
def test_sizes(M, N, K, wdt):
    i = SIZES.index((M, N, K))
    fn = FNS[i % 5]
    bias = [None, "f32", "bf16"][i % 3]
    res = [None, "bf16", "f32"][(i // 2) % 3]
    log(f"linear {M}x{N}x{K} {wdt} {fn} bias {bias} residual {res}")
    x, w, s, b, r = make(M, N, K, wdt, bias, res, seed=i)
    for out in {torch.float32, x.dtype}:
        y = aep.linear(x, w, scale=s, bias=b, activation=fn, residual=r, out_dtype=out)
        assert y.dtype == out and y.shape == (M, N)
        check(y, x, w, s, b, r, fn, (M, N, K, wdt, fn, out))


@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("wdt,out", [("bf16", "bf16"), ("bf16", "f32"), ("fp8", "bf16"), ("f32", "f32")])
def test_activations(fn, wdt, out):
    x, w, s, b, r = make(37, 203, 256, wdt, "f32", "bf16" if wdt != "f32" else "f32", seed=5)
    x = (x.float() * torch.linspace(0.01, 2.0, 37, device="cuda")[:, None]).to(x.dtype)  # saturated and not
    y = aep.linear(x, w, scale=s, bias=b, activation=fn, residual=r, out_dtype=TYPES[out])
    check(y, x, w, s, b, r, fn, (fn, wdt, out))


@pytest.mark.parametrize("pad,off", [(8, 0), (1, 0), (0, 1), (3, 5), (64, 8)])
@pytest.mark.parametrize("wdt", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("M,N,K", [(5, 40, 200), (70, 130, 264)])
def test_strides_and_offsets(pad, off, wdt, M, N, K):
    """Rows apart from each other, starting anywhere; what lies between them (NaN) is neither read into the
    result nor written."""
    x, w, s, b, r = make(M, N, K, wdt, "bf16", "f32", seed=7, pad=pad, off=off)
    dt = torch.float32 if wdt == "f32" else torch.bfloat16
    buf = torch.full((off + (M + 2) * (N + pad),), 77.0, dtype=dt, device="cuda")
    y = buf[off:].view(M + 2, N + pad)[1:M + 1, :N]
    got = aep.linear(x, w, scale=s, bias=b, activation="silu", residual=r, out=y)
    assert got is y
    check(y, x, w, s, b, r, "silu", (pad, off, wdt))
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[off:].view(M + 2, N + pad)[1:M + 1, :N] = False
    assert (buf[rest] == 77.0).all()


@pytest.mark.parametrize("M,N,K", [(3, 50, 128), (90, 200, 256)])
def test_residual_in_place(M, N, K):
    x, w, s, b, r = make(M, N, K, "bf16", "f32", "bf16", seed=9)
    keep = r.clone()
    y = aep.linear(x, w, bias=b, residual=r, out=r)
    assert y is r
    check(y, x, w, s, b, keep, "none", "in place")


def test_non_finite_values_stay_in_their_rows_and_columns():
    M, N, K = 70, 90, 130
    x, w, s, b, r = make(M, N, K, "bf16", None, None, seed=11)
    x[7, 129] = float("nan")
    x[20, 0] = float("inf")
    w[33, 5] = float("-inf")
    y = aep.linear(x, w, out_dtype=torch.float32)
    ref = x.double() @ w.double().T
    assert torch.equal(y.isnan(), ref.isnan())
    assert torch.equal(y.isinf(), ref.isinf()) and torch.equal(y[y.isinf()].double(), ref[ref.isinf()])


def test_empty_and_refusals():
    x, w, s, b, r = make(4, 16, 32, "bf16", "f32", None)
    assert aep.linear(x[:0], w, bias=b).shape == (0, 16)
    for bad in (dict(x=x.float()), dict(x=x.t()), dict(x=x[:, :31]), dict(x=x[:1].expand(4, 32)), dict(w=w.half()),
                dict(scale=torch.ones(16, dtype=torch.bfloat16, device="cuda")), dict(bias=b[:15]), dict(bias=b.cpu()),
                dict(residual=torch.zeros(4, 15, device="cuda")), dict(activation="tanh"), dict(x=x.cpu()),
                dict(out=torch.empty(4, 16, device="cuda")), dict(out_dtype=torch.float16), dict(w=w.view(-1))):
        a = dict(x=x, w=w, bias=b)
        a.update(bad)
        with pytest.raises(ValueError):
            aep.linear(a.pop("x"), a.pop("w"), **a)
    with pytest.raises(aep.AEPError):  # y is the residual, with another row stride
        buf = torch.zeros(4, 40, device="cuda", dtype=torch.bfloat16)
        aep.linear(x, w, residual=buf[:, :16], out=buf.view(-1)[:64].view(4, 16))


@pytest.mark.parametrize("M,N,K,wdt", [(3, 64, 512, "bf16"), (130, 300, 1024, "bf16"), (300, 520, 2048, "fp8")])
def test_streams_graphs_and_equal_bits(M, N, K, wdt):
    x, w, s, b, r = make(M, N, K, wdt, "f32", "bf16", seed=13)
    lin = aep.Linear(w, scale=s, bias=b, activation="gelu")
    ref = lin(x, r)
    check(ref, x, w, s, b, r, "gelu", "eager")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = lin(x, r)
    torch.cuda.synchronize()
    assert torch.equal(again, ref)
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
        # both at once, on streams of their own, and eager work beside them
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        mine = lin(x, r)
        torch.cuda.synchronize()
        assert all(torch.equal(o, ref) for o in outs) and torch.equal(mine, ref), i


def test_rows_far_apart():
    """Row offsets past 2^32 bytes."""
    K, N, ld = 128, 40, (1 << 31) + 8
    buf = torch.empty(2 * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, K), (ld, 1))
    x.copy_(torch.randn(2, K))
    _, w, _, b, _ = make(2, N, K, seed=15)
    y = aep.linear(x, w, bias=b)
    check(y, x, w, None, b, None, "none", "far x")
    w2 = buf.as_strided((2, K), (ld, 1))
    w2.copy_(torch.randn(2, K))
    x2 = make(3, 2, K, seed=16)[0]
    y = aep.linear(x2, w2)
    check(y, x2, w2, None, None, None, "none", "far w")
    out = buf.as_strided((2, N), (ld, 1), 4096)
    r = buf.as_strided((2, N), (ld, 1), 8192)
    r.copy_(torch.randn(2, N))
    x3 = make(2, N, K, seed=17)[0]
    aep.linear(x3, w, residual=r, out=out)
    check(out, x3, w, None, None, r, "none", "far y")
