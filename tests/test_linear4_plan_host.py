"""CPU: which kernel runs a dense product with 4-bit weights (linear4_cut.hip), and that the sizes of
the GPU tests take every one of them."""

import ctypes
import os
import subprocess

import pytest

import test_gpu_linear4 as gpu
from ffn_host import CLANG, CSRC, HERE


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("needs ROCm's clang++ as the host compiler")
    tmp = tmp_path_factory.mktemp("plan4")
    (tmp / "hip").mkdir()
    (tmp / "hip" / "hip_runtime.h").write_text("")
    so = str(tmp / "plan4.so")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-w", "-I", str(tmp), "-I", CSRC,
                    os.path.join(HERE, "linear4_plan_host.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.plan4.restype = ctypes.c_longlong
    lib.plan4.argtypes = [ctypes.c_int] * 3 + [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_void_p]

    def run(m, n, k, ldx=None, aligned=None, max_bytes=1 << 40):
        out = (ctypes.c_int * 4)()
        ldx = k if ldx is None else ldx
        b = lib.plan4(m, n, k, ldx, int(ldx % 8 == 0 if aligned is None else aligned), max_bytes, 256, out)
        return dict(widen=bool(out[0]), rf=out[1], cf=out[2], k8=out[3], bytes=b)

    return run


def test_small_products_take_small_tiles(plan):
    assert (plan(1, 4096, 4096)["rf"], plan(1, 4096, 4096)["cf"]) == (1, 1)
    assert (plan(1, 14336, 4096)["rf"], plan(1, 14336, 4096)["cf"]) == (1, 4)
    assert plan(777, 4096, 4096)["rf"] == 8 and not plan(777, 4096, 4096)["widen"]
    assert plan(2048, 4096, 4096)["widen"]
    for m, n, k in ((1, 1, 1), (1, 1, 1 << 21), (1 << 20, 7, 64), (1 << 30, 1, 1), (64, 1 << 20, 64)):
        c = plan(m, n, k)
        assert c["rf"] in (1, 2, 4, 8) and c["cf"] in (1, 2, 4, 8) and c["bytes"] >= 0


def test_scratch(plan):
    c = plan(2048, 4096, 4096)
    assert c["bytes"] >= 2 * 4096 * 4096
    assert plan(2048, 4096, 4096, aligned=False)["bytes"] >= c["bytes"] + 2 * 2048 * 4096
    assert not plan(2048, 4096, 4096, max_bytes=2 * 4096 * 4096 - 1)["widen"]
    # rows too far apart for 32-bit offsets: not the tile kernel's
    assert plan(777, 4096, 4096, ldx=1 << 22)["rf"] != 8


def test_gpu_tests_take_every_kernel(plan):
    tiles = {(plan(m, n, k)["rf"], plan(m, n, k)["cf"]) for m, n, k in gpu.SIZES}
    tiles |= {(plan(m, n, k)["rf"], plan(m, n, k)["cf"]) for m, n, k, _, _ in gpu.LARGE}
    assert tiles == {(1, 1), (1, 2), (1, 4), (2, 2), (2, 4), (4, 4)}
    for m, n, k, pad, off in gpu.TILE:
        c = plan(m, n, k, k + pad, off % 8 == 0 and (k + pad) % 8 == 0)
        assert c["rf"] == 8 and not c["widen"], (m, n, k)
    for m, n, k, pad, off in gpu.WIDE:
        assert plan(m, n, k, k + pad, off % 8 == 0 and (k + pad) % 8 == 0)["widen"], (m, n, k)
