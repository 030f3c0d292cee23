"""The dense product and routing, called as their documents allow: from several
threads at once, again and again with other work between, and on matrices of more
than 2^31 elements."""

import threading

import pytest
import torch

import paper_2505_08944_amd as aep
from gpu_helpers import log
from test_gpu_linear import TYPES

pytestmark = pytest.mark.gpu


def test_threads_on_streams_of_their_own():
    """One Linear (rows that are copied first, and rows that are not) and one Router."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def rnd(*s):
        return torch.randn(*s, device="cuda", generator=g)

    lin = aep.Linear(rnd(4104, 2731).to(torch.bfloat16), activation="gelu")
    xs = [rnd(m, 2731).to(torch.bfloat16) for m in (1, 33, 300, 900)]
    router = aep.Router(256, 8, score="sigmoid", n_groups=8, top_groups=4, group_top=2)
    logits, bias = [rnd(t, 256) for t in (1, 50, 3000)], torch.rand(256, device="cuda", generator=g)
    want = [lin(x) for x in xs], [aep.route(router, l, bias) for l in logits]
    torch.cuda.synchronize()
    bad = []

    def work(k):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for i in range(40):
                    y, (idx, w) = lin(xs[(i + k) % 4]), aep.route(router, logits[i % 3], bias)
                    st.synchronize()
                    if not (torch.equal(y, want[0][(i + k) % 4]) and torch.equal(idx, want[1][i % 3][0]) and
                            torch.equal(w, want[1][i % 3][1])):
                        bad.append((k, i))
        except Exception as e:  # (a thread's own would be lost)
            bad.append((k, repr(e)))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(5)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad[:4]


@pytest.mark.parametrize("M,N,K,wdt", [(1, 14336, 4096, "fp8"), (32, 4096, 4096, "bf16"), (256, 512, 256, "f32"),
                                       (777, 4096, 4096, "bf16")])
def test_equal_bits_again_and_again(M, N, K, wdt):
    g = torch.Generator(device="cuda").manual_seed(5)

    def call():
        act = torch.float32 if wdt == "f32" else torch.bfloat16
        w = (torch.randn(N, K, device="cuda", generator=g) * (50.0 if wdt == "fp8" else 0.5)).to(TYPES[wdt])
        s = (torch.rand(N, device="cuda", generator=g) * 0.02).to(torch.bfloat16) if wdt == "fp8" else None
        lin = aep.Linear(w, scale=s, bias=torch.randn(N, device="cuda", generator=g), activation="silu")
        return lin, torch.randn(M, K, device="cuda", generator=g).to(act)

    (a, x), (b, z) = call(), call()
    ref = a(x)
    for i in range(60):
        if i % 2:
            b(z)
        assert torch.equal(a(x), ref), i


@pytest.mark.parametrize("M,N,K,wdt,out,pad", [(70001, 32771, 136, "bf16", "bf16", 5), (40000, 57344, 128, "bf16", "f32", 0),
                                               (300, 600000, 4096, "fp8", "bf16", 0), (600000, 300, 4096, "bf16", "f32", 0),
                                               (3, 600001, 4099, "bf16", "bf16", 0)])
def test_more_than_31_bits_of_elements(M, N, K, wdt, out, pad):
    """Results, weights and tokens; rows from the start, the middle and the end, all columns."""
    log(f"linear {M}x{N}x{K} {wdt} {out}")
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.empty(M, K, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    w = torch.empty(N, K, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    s = None
    if wdt == "fp8":
        w = w.mul_(50.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
        s = torch.full((N,), 2.0 ** -6, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(M, N + pad, device="cuda", dtype=TYPES[out])[:, :N]
    aep.linear(x, w, scale=s, out=y, out_dtype=TYPES[out])
    rows = torch.arange(M) if M < 24 else torch.cat([torch.arange(8), torch.arange(M // 2, M // 2 + 8), torch.arange(M - 8, M)])
    rows = rows.cuda()
    xd = x[rows].double()
    for c in range(0, N, 65536):
        wd = w[c:c + 65536].double() * (2.0 ** -6 if s is not None else 1.0)
        ref, size = torch.nn.functional.linear(xd, wd), torch.nn.functional.linear(xd.abs(), wd.abs())
        # the sum's roundings and the result's (test_gpu_linear.py)
        tol = (K + 16) * 2.0 ** -23 * size
        tol = tol + (2.0 ** -8 if out == "bf16" else 2.0 ** -23) * (ref.abs() + tol)
        assert bool(((y[rows, c:c + 65536].double() - ref).abs() <= tol).all()), c
