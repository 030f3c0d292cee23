"""Operands of large products that start off 16 bytes are copied to aligned rows,
through the binding as with scratch given by hand."""

import ctypes

import pytest
import torch

import paper_2505_08944_amd as aep
from gpu_helpers import log
from paper_2505_08944_amd import _lib as L
from test_gpu_linear import TYPES
from test_gpu_linear_tiles import gpu_check

pytestmark = pytest.mark.gpu


def shifted(t, off):
    """t's values from `off` elements past an aligned address on."""
    buf = torch.full((t.numel() + 32,), float("nan"), device="cuda").to(t.dtype)
    v = buf[off:off + t.numel()].view(t.shape)
    v.copy_(t)
    return v


def operands(M, N, K, wdt):
    x = torch.randn(M, K, device="cuda").to(torch.bfloat16)
    w = (torch.randn(N, K, device="cuda") * (50.0 if wdt == "fp8" else 0.5)).to(TYPES[wdt])
    s = (torch.rand(N, device="cuda") * 0.02 + 0.001).to(torch.bfloat16) if wdt == "fp8" else None
    return x, w, s, torch.randn(N, device="cuda")


@pytest.mark.parametrize("M,N,K,wdt", [(2048, 4096, 4096, "bf16"), (1100, 4104, 1024, "bf16"), (1100, 4104, 2048, "fp8")])
def test_the_binding_gives_room_for_copies(M, N, K, wdt):
    """The copies are the aligned operands, so the sums are the same in every bit: f32
    results, which another kernel's order of sums would change."""
    torch.manual_seed(31)
    x, w, s, b = operands(M, N, K, wdt)
    ref = aep.linear(x, w, scale=s, bias=b, activation="silu", out_dtype=torch.float32)
    gpu_check(ref, x, w, s, b, None, "silu", "aligned")
    lin = aep.Linear(w, scale=s, bias=b, activation="silu", out_dtype=torch.float32)
    for xo, wo in ((1, 0), (4, 0), (0, 1), (3, 5), (0, 0), (1, 0)):
        log(f"copies {M}x{N}x{K} {wdt} x {xo} w {wo}")
        xs, ws = shifted(x, xo), shifted(w, wo)
        assert torch.equal(aep.linear(xs, ws, scale=s, bias=b, activation="silu", out_dtype=torch.float32), ref), (xo, wo)
        assert torch.equal(lin(xs), ref), xo  # one Linear, x of one alignment after another


def region_written(ws, lo, n):
    return not bool((ws[lo:lo + n] == 255).all())


@pytest.mark.parametrize("M,N,K,wdt", [(1100, 4104, 1024, "bf16"), (1100, 4104, 2048, "fp8"), (1000, 5000, 2731, "bf16"),
                                       (777, 2003, 2001, "bf16")])
def test_which_operands_are_copied(M, N, K, wdt):
    """The copies lie behind the pieces' sums: x's, then W's, each written where its operand is not
    aligned, and only there."""
    torch.manual_seed(33)
    x, w, s, b = operands(M, N, K, wdt)
    lib, need, sums = L.lib(), ctypes.c_size_t(), ctypes.c_size_t()
    es = 1 if wdt == "fp8" else 2
    whole = -(-K // (16 // es)) * (16 // es)  # K of the copies
    rows_off = K != whole

    def desc(k):
        return L.LinearDesc(M, N, k, L.AEP_BF16, L.AEP_FP8_E4M3 if wdt == "fp8" else L.AEP_BF16, L.AEP_BF16, L.AEP_F32,
                            L.AEP_BF16, L.AEP_FN_GELU, k, k, N, N)

    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    d, aligned = desc(K), desc(whole)
    for xo, wo in ((0, 0), (1, 0), (0, 1), (3, 2)):
        xs, ws_ = shifted(x, xo), shifted(w, wo)
        log(f"copied operands {M}x{N}x{K} {wdt} x {xo} w {wo}")
        assert lib.aep_linear_workspace_at(ctypes.byref(d), xs.data_ptr(), ws_.data_ptr(), None, y.data_ptr(),
                                           ctypes.byref(need)) == 0
        xb, wb = (M * whole * 2 if xo or rows_off else 0), (N * whole * es if wo or rows_off else 0)
        n = need.value
        assert lib.aep_linear_workspace_at(ctypes.byref(aligned), 1 << 20, 1 << 20, None, y.data_ptr(),
                                           ctypes.byref(sums)) == 0
        # the same product of aligned rows has the same cut, whose sums come first
        assert n == sums.value + xb + wb
        scratch = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")
        assert lib.aep_linear(ctypes.byref(d), xs.data_ptr(), ws_.data_ptr(), None if s is None else s.data_ptr(),
                              b.data_ptr(), None, y.data_ptr(), scratch.data_ptr() if n else None, n,
                              torch.cuda.current_stream().cuda_stream) == 0
        gpu_check(y, x, w, s, b, None, "gelu", (xo, wo))
        assert bool((scratch[n:] == 255).all())
        at = sums.value
        for bytes_, values, rows in ((xb, x, M), (wb, w, N)):
            if bytes_:
                copy = scratch[at:at + bytes_].view(values.dtype).view(rows, whole)
                assert torch.equal(copy[:, :K].float(), values.float())
                assert not copy[:, K:].float().any()
            at += bytes_
