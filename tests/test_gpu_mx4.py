"""The quantiser against a 64-bit search for the nearest code: equal codes, scales and values."""

import numpy as np
import pytest
import torch

import mx4_ref
import paper_2505_08944_amd as aep
from gpu_helpers import log

pytestmark = pytest.mark.gpu


def check(x):
    """Codes, scales and values of a device matrix."""
    codes, scale = aep.quantize_mx4(x)
    code, want_scale, want = mx4_ref.quantize(x.double().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    bad = np.repeat(want_scale == 255, 32, -1)[:, :x.shape[1]]
    got = codes.cpu().numpy()
    each = np.stack([got & 15, got >> 4], -1).reshape(got.shape[0], -1)
    assert np.array_equal(each[:, :x.shape[1]][~bad], code[~bad])
    if x.shape[1] % 2:
        assert (each[:, -1] == 0).all()
    for dtype in (torch.bfloat16, torch.float32):
        y = aep.dequantize_mx4(codes, scale, x.shape[1], dtype=dtype)
        assert y.dtype == dtype
        assert np.array_equal(y.double().cpu().numpy(), want, equal_nan=True)
    return codes, scale


@pytest.mark.parametrize("n,k", [(1, 1), (1, 2), (3, 7), (2, 31), (5, 32), (4, 33), (7, 64), (3, 95), (130, 257), (2, 4096),
                                 (513, 40), (1, 100001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sizes(n, k, dtype):
    log(f"quantize {n} x {k} {dtype}")
    g = torch.Generator().manual_seed(n * 7 + k)
    x = torch.randn(n, k, generator=g) * torch.exp2(torch.randint(-20, 20, (n, 1), generator=g).float())
    check(x.to(dtype).cuda())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_middles_and_borders(dtype):
    """Values in the middle between codes and beside it, blocks whose largest value is at a power's border, at every
    power of the type, subnormal ones, zeros of both signs."""
    step = 2.0 ** -23 if dtype == torch.float32 else 2.0 ** -7
    mids = np.array([0.0, -0.0, 0.25, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 4.0])
    rows = []
    for top in (7.0, 7.0 * (1 - step), 7.0 * (1 + step), 8.0, 4.0, 3.5, 6.0, 1.0):
        for e in [-145, -133, -130, -127, -126, -125, -100, -9, 0, 5, 60, 120, 124]:
            r = np.concatenate([mids, -mids[:8], mids[:5] * (1 + step), mids[3:9] * (1 - step), [top]])
            rows.append(np.ldexp(r, e))
    x = torch.from_numpy(np.array(rows)).to(dtype)
    x[torch.isinf(x)] = 0.0
    check(x.cuda())
    check(torch.zeros(3, 70, dtype=dtype).cuda())
    check(torch.full((2, 40), torch.finfo(dtype).max, dtype=dtype).cuda())


def test_blocks_that_are_not_finite():
    x = torch.randn(6, 100)
    x[0, 3], x[1, 40], x[2, 99], x[3, 64] = float("nan"), float("inf"), -float("inf"), float("nan")
    for dtype in (torch.float32, torch.bfloat16):
        check(x.to(dtype).cuda())


def test_strides():
    x = torch.randn(9, 203).cuda()
    for dtype in (torch.float32, torch.bfloat16):
        y = x.to(dtype)
        check(y[:, 1:78])
        check(y[::2, 3:100])
    codes, scale = aep.quantize_mx4(x)
    out = torch.full((9, 300), 7.0, device="cuda")
    aep.dequantize_mx4(codes, scale, 203, dtype=torch.float32, out=out[:, 5:208])
    assert torch.equal(out[:, 5:208], aep.dequantize_mx4(codes, scale, 203, dtype=torch.float32))
    assert (out[:, :5] == 7).all() and (out[:, 208:] == 7).all()


def test_every_code_and_scale():
    """All 16 codes under all 256 scales (the largest value of the largest power is beyond both types: infinity)."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).cuda()
    scale = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 16).cuda()
    got = codes.cpu().numpy()
    each = np.stack([got & 15, got >> 4], -1).reshape(256, -1)
    want = mx4_ref.values(each, scale.cpu().numpy())
    want[np.abs(want) > 3.4e38] = np.inf * np.sign(want[np.abs(want) > 3.4e38])
    for dtype in (torch.bfloat16, torch.float32):
        y = aep.dequantize_mx4(codes.view(torch.float4_e2m1fn_x2), scale.view(torch.float8_e8m0fnu), 512, dtype=dtype)
        assert np.array_equal(y.double().cpu().numpy(), want, equal_nan=True)


def test_no_rows():
    codes, scale = aep.quantize_mx4(torch.empty(0, 50, device="cuda"))
    assert codes.shape == (0, 25) and scale.shape == (0, 2)
    assert aep.dequantize_mx4(codes, scale, 50).shape == (0, 50)


def test_more_than_32_bits_of_values():
    n, k = 70001, 65536
    log(f"quantize {n} x {k}")
    x = torch.empty(n, k, device="cuda", dtype=torch.bfloat16)
    x.view(-1)[:1 << 20].normal_()
    x[1:] = x[0]
    x[-1] = -x[0]
    codes, scale = aep.quantize_mx4(x)
    want_c, want_s = aep.quantize_mx4(x[:1])
    assert bool((scale == want_s).all())
    assert bool((codes[:-1] == want_c).all()) and bool((codes[-1] == want_c ^ 0x88).all())
    del x
    y = aep.dequantize_mx4(codes, scale, k)
    one = aep.dequantize_mx4(want_c, want_s, k)
    assert bool((y[:-1] == one).all()) and bool((y[-1] == -one).all())


def test_a_number_of_columns_in_a_tensor_counts_by_its_value():
    x = torch.randn(3, 40, generator=torch.Generator().manual_seed(3)).cuda()
    codes, scale = aep.quantize_mx4(x)
    want = aep.dequantize_mx4(codes, scale, 40)
    k = torch.tensor(40)
    assert torch.equal(aep.dequantize_mx4(codes, scale, k), want)
    k.fill_(39)
    assert torch.equal(aep.dequantize_mx4(codes, scale, k), want[:, :39])
    k.fill_(400)
    for bad in (k, 40.0, 1 << 40, 0):
        for _ in range(2):
            with pytest.raises((TypeError, ValueError, aep.AEPError)):
                aep.dequantize_mx4(codes, scale, bad)
