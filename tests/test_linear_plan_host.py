"""CPU: which kernel runs a dense product and how its tiles are cut
(linear_cut.hip), and that the sizes of the GPU tests are cut every way there is."""

import ctypes
import itertools
import os
import subprocess

import pytest

import test_gpu_linear_tiles as gpu
from ffn_host import CLANG, CSRC, HERE


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("needs ROCm's clang++ as the host compiler")
    tmp = tmp_path_factory.mktemp("plan")
    (tmp / "hip").mkdir()
    (tmp / "hip" / "hip_runtime.h").write_text("")
    so = str(tmp / "plan.so")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-w", "-I", str(tmp), "-I", CSRC,
                    os.path.join(HERE, "linear_plan_host.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.plan.argtypes = [ctypes.c_int] * 6 + [ctypes.c_longlong, ctypes.c_void_p, ctypes.c_void_p]
    names = ("tiles", "whole", "rest", "halves", "p0", "fam", "pr", "lrow", "items", "nrow", "ncol", "rf", "cf")

    def run(m, n, k, fp8=False, wide=True, max_floats=1 << 40, nwg=256):
        out, us = (ctypes.c_int * 13)(), (ctypes.c_double * 3)()
        lib.plan(m, n, k, int(fp8), int(wide), nwg, max_floats, out, us)
        return dict(zip(names, out), us=us[0], rows_us=us[1], floats=int(us[2]))

    return run


SHAPES = list(itertools.product((1, 33, 64, 65, 128, 129, 255, 256, 257, 385, 777, 1024, 4100, 20000),
                                (1, 8, 127, 128, 129, 256, 1000, 4096, 14336), (1, 64, 100, 1024, 4096, 14336)))


@pytest.mark.parametrize("fp8", [False, True])
def test_every_row_and_column_is_covered(plan, fp8):
    for m, n, k in SHAPES:
        c = plan(m, n, k, fp8)
        high = 256 >> c["fam"]
        covered = c["nrow"] * 256 + c["lrow"] * high
        assert covered >= m and (c["nrow"] - 1) * 256 < m and (c["nrow"] + 1) * 256 > m - c["lrow"] * high, (m, n, c)
        if c["lrow"]:
            assert c["fam"] in (1, 2) and c["nrow"] * 256 + (c["lrow"] - 1) * high < m, (m, n, c)
        assert c["ncol"] == -(-n // 256)
        assert c["whole"] + c["rest"] == c["nrow"] * c["ncol"] and c["whole"] % 256 == 0 and c["rest"] < 256
        last = c["lrow"] * -(-n // 128)
        assert c["items"] == c["whole"] + c["rest"] * c["halves"] * c["p0"] + last * c["pr"]
        steps = -(-k // 64)
        for p in (c["p0"], c["pr"]):
            assert 1 <= p <= 8 and (p == 1 or steps >= 4 * p), (m, n, k, c)
        want = (c["rest"] * c["halves"] * c["p0"] * (65536 // c["halves"]) if c["p0"] > 1 else 0) + \
            (last * c["pr"] * (32768 >> c["fam"]) if c["pr"] > 1 else 0)
        assert c["floats"] == want <= 24 << 20


def test_scratch_is_never_exceeded(plan):
    for m, n, k in SHAPES:
        for cap in (0, 1000, 1 << 20):
            assert plan(m, n, k, max_floats=cap)["floats"] <= cap


def test_the_faster_kernel_is_taken(plan):
    """us measured with both kernels, operands in the Infinity Cache."""
    for m, n, k, rows, tiles in ((128, 4096, 4096, 12.9, 20.4), (384, 4096, 4096, 29.9, 26.9), (777, 4096, 4096, 65, 39),
                                 (2048, 1024, 1024, 15.2, 16.3), (96, 14336, 4096, 31.9, 28.6), (512, 256, 7168, 12, 25),
                                 (2048, 4096, 4096, 160, 47), (8192, 64, 2048, 9, 24), (192, 4096, 14336, 63.7, 39.7)):
        c = plan(m, n, k)
        assert c["tiles"] == (tiles < rows), (m, n, k, c)
        assert abs(c["rows_us"] - rows) < 0.35 * rows + 1.5, (m, n, k, c)
    assert not plan(32, 4096, 4096)["tiles"] and not plan(1, 14336, 4096, True)["tiles"]


@pytest.mark.parametrize("fp8", [False, True])
def test_the_gpu_tests_cover_every_cut(plan, fp8):
    seen = set()
    for m, n, k in gpu.SIZES:
        c = plan(m, n, (k + 15) // 16 * 16 if fp8 else k, fp8)
        assert c["tiles"] or fp8, (m, n, k, c)
        if not c["tiles"]:
            continue
        if c["whole"]:
            seen.add("whole")
        if c["rest"]:
            seen.add(("rest", c["halves"], c["p0"] > 1))
        if c["fam"]:
            seen.add(("last", c["fam"], c["lrow"] > 1, c["pr"] > 1))
        if -(-n // 128) % 2 and c["rest"] and c["halves"] == 2:
            seen.add("odd halves")
    want = {"whole", "odd halves", ("rest", 1, False), ("rest", 2, False), ("rest", 2, True), ("last", 1, True, False),
            ("last", 1, True, True), ("last", 1, False, False), ("last", 2, False, False)}
    want |= set() if fp8 else {("last", 2, True, False), ("last", 2, True, True), ("last", 2, False, True)}
    assert want <= seen, want - seen
