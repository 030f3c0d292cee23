"""Builds the device code of the tiled dense product for the host, its LDS
accesses handed to the recorder that ffn_host.cpp has for the FFN's."""

import ctypes
import os
import re
import subprocess

import pytest

from ffn_host import CLANG, CSRC, HERE


def _device_part():
    """k_linear_tiles.hip up to its kernels, LDS accesses as recorder calls."""
    src = open(os.path.join(CSRC, "k_linear_tiles.hip")).read()
    head, rest = src.split("template <bool FP8>\n__global__", 1)
    assert "<<<" not in head and "<<<" in rest

    def sub(pattern, repl, text, n, flags=0):
        out, k = re.subn(pattern, repl, text, flags=flags)
        assert k == n if n else k > 0, (pattern, k)
        return out

    head = sub(r'asm volatile\("s_mov_b32 m0.*?\);', "lds_load(lds_addr);", head, 1, re.S)
    head = sub(r'asm volatile\("".*?\);', ";", head, 0)
    head = sub(r"\*reinterpret_cast<const (bf16x8_t|uint4)\*>\(q", r"lds_read<\1>(q", head, 3)
    assert "asm" not in re.sub(r"//.*", "", head)
    return head + "\n}  // namespace aep\n"


def load(tmp):
    if not os.path.exists(CLANG):
        pytest.skip("needs ROCm's clang++ as the host compiler")
    (tmp / "hip").mkdir()
    (tmp / "hip" / "hip_runtime.h").write_text("")  # the mock stands in for it
    mock = open(os.path.join(HERE, "ffn_host.cpp")).read().split('#include "ffn_device.inc"')[0]
    (tmp / "recorder.inc").write_text(mock)
    (tmp / "linear_device.inc").write_text(_device_part())
    so = str(tmp / "linear_host.so")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-w", "-I", str(tmp), "-I", CSRC,
                    os.path.join(HERE, "linear_host.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.linear_order_violations.restype = ctypes.c_long
    return lib
