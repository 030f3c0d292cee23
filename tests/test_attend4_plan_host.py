"""CPU: which kernels run the attention over the cache in 4 bits (attend4_plan.h), and that the GPU tests run all of them."""

import ctypes
import os
import subprocess

import pytest

import test_gpu_attend4 as gpu
from ffn_host import CLANG, CSRC, HERE


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("needs ROCm's clang++ as the host compiler")
    so = str(tmp_path_factory.mktemp("attend4") / "plan.so")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-w", "-I", CSRC,
                    os.path.join(HERE, "attend4_plan_host.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.plan.restype = ctypes.c_longlong
    lib.plan.argtypes = [ctypes.c_int] * 7 + [ctypes.c_longlong, ctypes.c_int, ctypes.c_void_p]

    def run(batch, total, heads, group, d, max_len, rows=False, max_rows=None):
        out = (ctypes.c_int * 9)()
        b = lib.plan(batch, total, rows, total if max_rows is None else max_rows, heads, group, d, max_len, 256, out)
        return b, [dict(zip(("nc", "workers", "over", "most"), out[1 + 4 * i:5 + 4 * i])) for i in range(out[0])]

    return run


def test_every_number_of_columns_is_taken_once(plan):
    for d in (64, 128, 256):
        for rows in (False, True):
            for batch, total, heads, group, max_len in ((1, 1, 1, 1, 0), (64, 64, 8, 4, 8192), (4, 2036, 8, 4, 8192),
                                                        (64, 575, 8, 4, 8192), (1, 1 << 20, 1, 1, 1 << 20), (1000, 1000, 1, 64, 64),
                                                        (3, 300, 2, 17, 1 << 17)):
                b, passes = plan(batch, total, heads, group, d, max_len, rows)
                assert passes[0]["over"] == 0 and passes[-1]["most"] == 2 ** 31 - 1
                assert len(passes) == 1 or passes[0]["most"] == passes[1]["over"]
                for p in passes:
                    assert p["nc"] in (1, 2, 8) and p["workers"] % 8 == 0 and 8 <= p["workers"] <= 1024
                    assert b >= p["workers"] * (2 * 16 * p["nc"] * (d + 2) * 4 + 32)


def test_kinds(plan):
    assert [p["nc"] for p in plan(64, 64, 8, 4, 128, 16384)[1]] == [1]
    assert [p["nc"] for p in plan(16, 80, 16, 1, 64, 2048)[1]] == [1]
    assert [p["nc"] for p in plan(32, 32 * 8, 4, 4, 128, 8192)[1]] == [2]
    assert [p["nc"] for p in plan(4, 2036, 8, 4, 128, 8192)[1]] == [8]
    assert [p["nc"] for p in plan(64, 575, 8, 4, 128, 8192, True)[1]] == [1, 8]
    assert [p["nc"] for p in plan(64, 64, 8, 4, 128, 8192, True, 1)[1]] == [1]


def test_gpu_tests_run_every_kernel(plan):
    seen = set()
    for lens, n, heads, group, d, page in gpu.CASES:
        total = n * len(lens) if isinstance(n, int) else sum(n)
        rows = not isinstance(n, int)
        tokens = max(max(1, -(-max(lens) // page)), 8 * 512 * 128 // (heads * len(lens)) // page + 1) * page
        _, passes = plan(len(lens), total, heads, group, d, tokens, rows)
        most = max([n] if isinstance(n, int) else n) * group
        seen |= {(d, p["nc"]) for p in passes if most > p["over"]}
    assert seen == {(d, nc) for d in (64, 128, 256) for nc in (1, 2, 8)}, seen
