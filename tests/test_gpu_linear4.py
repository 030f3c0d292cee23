"""aep_linear4 against a 64-bit product of the values that the codes stand for, element by element.

Tolerance: these are the bf16 values themselves, so it is that of a bf16 product (test_gpu_linear.py)."""

import threading

import numpy as np
import pytest
import torch

import mx4_ref
import ops_ref
import paper_2505_08944_amd as aep
from gpu_helpers import log
from test_gpu_linear import FNS, TYPES, f64

pytestmark = pytest.mark.gpu


def make(M, N, K, bias="f32", res="bf16", seed=0, pad=0, off=0):
    """(x, Linear4's codes and scale, 64-bit weights, bias, residual); pad, off: NaN between x's rows and before them."""
    g = torch.Generator().manual_seed(seed)

    def mat(r, c, dtype):
        t = torch.full((off + r * (c + pad),), float("nan"))
        t[off:].view(r, c + pad)[:, :c].copy_(torch.randn(r, c, generator=g))
        return t.to(dtype).cuda()[off:].view(r, c + pad)[:, :c]

    code = torch.randint(0, 16, (N, K), generator=g).numpy()
    scale = torch.randint(122, 127, (N, -(-K // 32)), generator=g).to(torch.uint8)
    w = mx4_ref.values(code, scale.numpy())
    return (mat(M, K, torch.bfloat16), torch.from_numpy(mx4_ref.pack(code)).cuda(), scale.cuda(), w,
            torch.randn(N, generator=g).to(TYPES[bias]).cuda() if bias else None, mat(M, N, TYPES[res]) if res else None)


def check(y, x, w, b, r, fn, what):
    ref, size = ops_ref.linear(f64(x), w, None, f64(b), fn, f64(r))
    K = x.shape[1]
    v = ref if r is None else ref - f64(r)
    tol = 1.13 * (K + 16) * 2.0 ** -23 * size + 2.0 ** -20 * np.abs(v) + 2.0 ** -24 * size
    if fn == "gelu":
        tol = tol + 2.0 ** -24 * size
    tol = tol + (2.0 ** -8 if y.dtype == torch.bfloat16 else 2.0 ** -23) * (np.abs(ref) + tol)
    got = f64(y)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], tol[bad][:4])


SIZES = [(1, 1, 1), (1, 1, 31), (1, 16, 64), (2, 7, 33), (1, 130, 512), (16, 16, 128), (17, 65, 72), (15, 64, 2048),
         (32, 64, 129), (33, 48, 1000), (48, 100, 65), (64, 256, 320), (65, 129, 96), (100, 300, 1027), (130, 70, 63),
         (200, 257, 520), (257, 513, 192), (4, 1000, 1153), (64, 1040, 3000), (3, 33, 5001)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(M, N, K):
    i = SIZES.index((M, N, K))
    fn, bias, res = FNS[i % 5], [None, "f32", "bf16"][i % 3], [None, "bf16", "f32"][(i // 2) % 3]
    log(f"linear4 {M}x{N}x{K} {fn} bias {bias} residual {res}")
    x, codes, scale, w, b, r = make(M, N, K, bias, res, seed=i)
    for out in (torch.float32, torch.bfloat16):
        lin = aep.Linear4(codes, scale, K, bias=b, activation=fn, out_dtype=out)
        y = lin(x, r)
        assert y.dtype == out and y.shape == (M, N)
        check(y, x, w, b, r, fn, (M, N, K, fn, out))


# larger ones, by the kernel that takes them: rows (tiles of all sizes); the tile kernel; weights widened first.  Whole
# tiles, rows and channels left over, K off 8 and off 128, x off 16 bytes
LARGE = [(16, 14336, 520, 0, 0), (40, 9000, 640, 0, 0), (64, 8200, 1000, 0, 0), (130, 4096, 1100, 0, 0), (256, 4096, 2048, 0, 0),
         (100, 14000, 300, 3, 1)]
TILE = [(777, 4096, 4096, 0, 0), (890, 4090, 4001, 0, 0), (1000, 4090, 4232, 8, 5), (640, 6001, 4100, 3, 0)]
WIDE = [(2048, 4096, 4096, 0, 0), (4096, 1408, 2048, 0, 0), (2304, 4104, 4001, 3, 1), (2048, 4096, 4104, 0, 5)]


@pytest.mark.parametrize("M,N,K,pad,off", LARGE + TILE + WIDE)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_large(M, N, K, pad, off, out):
    log(f"linear4 {M}x{N}x{K} pad {pad} off {off} {out}")
    x, codes, scale, w, b, r = make(M, N, K, "f32", "bf16", seed=M + K, pad=pad, off=off)
    y = aep.Linear4(codes, scale, K, bias=b, activation="silu", out_dtype=out)(x, r)
    assert bool(torch.isfinite(y).all())
    # (rows enough for the check: a tile's first and last ones, and the last)
    rows = torch.tensor(sorted({0, 1, 15} | {i for i in (63, 64, 127, 128, 255, 256, 300) if i < M} | {M // 2, M - 2, M - 1}))
    check(y[rows], x[rows], w, b, r[rows], "silu", (M, N, K, pad, off))


@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_activations(fn, out):
    x, codes, scale, w, b, r = make(37, 203, 256, seed=5)
    x = (x.float() * torch.linspace(0.01, 2.0, 37, device="cuda")[:, None]).to(x.dtype)  # saturated and not
    check(aep.Linear4(codes, scale, bias=b, activation=fn, out_dtype=out)(x, r), x, w, b, r, fn, (fn, out))


@pytest.mark.parametrize("pad,off", [(8, 0), (1, 0), (0, 1), (3, 5), (64, 8)])
@pytest.mark.parametrize("M,N,K", [(5, 40, 200), (70, 130, 264)])
def test_strides_and_offsets(pad, off, M, N, K):
    """What lies between rows (NaN) is neither read into the result nor written."""
    x, codes, scale, w, b, r = make(M, N, K, "bf16", "f32", seed=7, pad=pad, off=off)
    buf = torch.full((off + (M + 2) * (N + pad),), 77.0, dtype=torch.bfloat16, device="cuda")
    y = buf[off:].view(M + 2, N + pad)[1:M + 1, :N]
    lin = aep.Linear4(codes, scale, K, bias=b, activation="silu")
    assert lin(x, r, y) is y
    check(y, x, w, b, r, "silu", (pad, off))
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[off:].view(M + 2, N + pad)[1:M + 1, :N] = False
    assert (buf[rest] == 77.0).all()


def test_residual_in_place_and_values_that_are_not_finite():
    x, codes, scale, w, b, r = make(9, 50, 160, seed=9)
    keep = r.clone()
    lin = aep.Linear4(codes, scale, bias=b)
    assert lin(x, r, r) is r
    check(r, x, w, b, keep, "none", "in place")
    # a NaN row of x, and a block of W without a value, reach their own results alone
    x[4, 3] = float("nan")
    scale[7, 2] = 255
    y = aep.Linear4(codes, scale, bias=b)(x)
    bad = torch.isnan(y)
    assert bad[4].all() and bad[:, 7].all() and int(bad.sum()) == 50 + 9 - 1


def test_codes_are_laid_out_once():
    x, codes, scale, w, b, _ = make(4, 70, 100, seed=2)
    lin = aep.Linear4(codes.view(torch.float4_e2m1fn_x2), scale.view(torch.float8_e8m0fnu), 100, bias=b)
    y = lin(x)
    codes.zero_()
    assert torch.equal(lin(x), y)
    b.add_(1.0)  # (the bias is the caller's)
    check(lin(x), x, w, b, None, "none", "bias")


def test_little_scratch():
    """The C call with less scratch than asked for, and none: as right."""
    import ctypes

    from paper_2505_08944_amd import _lib as L
    x, codes, scale, w, b, r = make(2048, 4096, 4096, seed=4)
    lin, y = aep.Linear4(codes, scale, bias=b), torch.empty(2048, 4096, dtype=torch.bfloat16, device="cuda")
    d = L.Linear4Desc(2048, 4096, 4096, L.AEP_BF16, L.AEP_F32, L.AEP_BF16, 0, 4096, 4096, 4096)
    need = ctypes.c_size_t()
    assert L.lib().aep_linear4_workspace(ctypes.byref(d), x.data_ptr(), None, 16, ctypes.byref(need)) == 0
    assert need.value >= 2 * 4096 * 4096
    for size in (need.value, need.value - 16, 2 * 4096 * 4096, 2 * 4096 * 4096 - 1, 0):
        ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
        assert L.lib().aep_linear4(ctypes.byref(d), x.data_ptr(), lin.packed.data_ptr(), b.data_ptr(), None, y.data_ptr(),
                                   ws.data_ptr() if size else None, size, L.raw_stream(0)) == 0
        check(y[:40], x[:40], w, b, None, "none", size)


def test_streams_threads_and_graphs():
    """One Linear4 from several threads, each on its stream; captured and replayed beside eager calls."""
    x, codes, scale, w, b, _ = make(900, 2056, 1027, seed=6)
    lin = aep.Linear4(codes, scale, 1027, bias=b)
    xs = [x[:m] for m in (1, 33, 300, 900)]
    want = [lin(t) for t in xs]
    check(want[1], xs[1], w, b, None, "none", "33 rows")
    torch.cuda.synchronize()
    bad = []

    def work(k):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for i in range(30):
                    y = lin(xs[(i + k) % 4])
                    st.synchronize()
                    if not torch.equal(y, want[(i + k) % 4]):
                        bad.append((k, i))
        except Exception as e:  # (a thread's own would be lost)
            bad.append((k, repr(e)))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad[:4]
    outs = [torch.empty_like(t) for t in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for t, o in zip(xs, outs):
            lin(t, None, o)
    for i in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, t) for o, t in zip(outs, want)), i
        assert torch.equal(lin(xs[2]), want[2])


def test_no_rows():
    x, codes, scale, w, b, _ = make(1, 20, 64, seed=1)
    assert aep.Linear4(codes, scale)(x[:0]).shape == (0, 20)


def test_more_than_31_bits_of_weights():
    n, k = 600001, 8192
    log(f"linear4 3 x {n} x {k}")
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (n, k // 2), device="cuda", generator=g, dtype=torch.uint8)
    scale = torch.randint(120, 127, (n, k // 32), device="cuda", generator=g, dtype=torch.uint8)
    x = torch.randn(3, k, device="cuda", generator=g).to(torch.bfloat16)
    y = aep.Linear4(codes, scale)(x)
    for c in (0, n // 2, n - 300):
        w = aep.dequantize_mx4(codes[c:c + 300], scale[c:c + 300], k, dtype=torch.float32).double()
        ref, size = x.double() @ w.T, x.double().abs() @ w.abs().T
        tol = (k + 16) * 2.0 ** -23 * size
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
        assert bool(((y[:, c:c + 300].double() - ref).abs() <= tol).all()), c
