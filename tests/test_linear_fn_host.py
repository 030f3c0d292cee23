"""CPU: the activations' own errors, by value, against 64 bits (aep.h states them):
f32 results 2^-20 of their value and 2^-142; bf16 results, before their rounding, 2^-15, GELU by
2^-23 |v| more, and results below 2^-119 may be lost.  (2^-142: the exponential has steps
of 2^-149 at least, half of one times |v| below 110.)"""

import ctypes
import os
import subprocess

import numpy as np
import pytest

import ops_ref
from ffn_host import CLANG, CSRC, HERE

FNS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def act(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("needs ROCm's clang++ as the host compiler")
    tmp = tmp_path_factory.mktemp("fn")
    (tmp / "hip").mkdir()
    (tmp / "hip" / "hip_runtime.h").write_text("")
    so = str(tmp / "fn.so")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-shared", "-fPIC", "-w", "-I", str(tmp), "-I", CSRC,
                    "-I", os.path.join(os.path.dirname(HERE), "include"), os.path.join(HERE, "linear_fn_host.cpp"), "-o",
                    so], check=True)
    lib = ctypes.CDLL(so)
    lib.activations.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_long]

    def run(exact, fn, v):
        v = np.ascontiguousarray(v, np.float32)
        y = np.empty_like(v)
        lib.activations(int(exact), FNS.index(fn), v.ctypes.data, y.ctypes.data, v.size)
        return y

    return run


def arguments():
    g = np.random.default_rng(1)
    small = np.float32(2.0) ** np.arange(-149, 10).astype(np.float32)
    return np.concatenate([np.linspace(-110, 30, 60001), np.linspace(-6, 6, 20001), g.standard_normal(20000), small, -small,
                           [0.0, -0.0, 1e10, -1e10, 1e30, -1e30, 3e38, -3e38]]).astype(np.float32)


def reference(fn, v):
    with np.errstate(over="ignore", invalid="ignore"):
        if fn == "gelu_tanh":  # by its form without the cancellation of 1 + tanh
            u = 2.0 * np.sqrt(2.0 / np.pi) * (v + 0.044715 * v ** 3)
            return v / (1.0 + np.exp(-u))
        return ops_ref.linear_fn(fn, v)


@pytest.mark.parametrize("fn", FNS)
def test_f32_results(act, fn):
    v = arguments()
    ref = reference(fn, v.astype(np.float64))
    bad = ~(np.abs(act(True, fn, v) - ref) <= 2.0 ** -20 * np.abs(ref) + 2.0 ** -142)
    assert not bad.any(), (fn, int(bad.sum()), v[bad][:5], act(True, fn, v)[bad][:5], ref[bad][:5])


@pytest.mark.parametrize("fn", FNS)
def test_bf16_results(act, fn):
    v = arguments()
    ref = reference(fn, v.astype(np.float64))
    tol = 2.0 ** -15 * np.abs(ref) + 2.0 ** -119
    if fn == "gelu":
        tol = tol + 2.0 ** -23 * np.abs(v)
    bad = ~(np.abs(act(False, fn, v) - ref) <= tol)
    assert not bad.any(), (fn, int(bad.sum()), v[bad][:5], act(False, fn, v)[bad][:5], ref[bad][:5])


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("fn", FNS)
def test_values_that_are_not_finite(act, fn, exact):
    got = act(exact, fn, [np.nan, np.inf, -np.inf])
    assert np.isnan(got[0]) and got[1] == np.inf
    if fn == "relu":
        assert got[2] == 0
    elif fn == "none":
        assert got[2] == -np.inf
    else:  # the limit is 0, the formulas' -inf times 0 is not a number: either, but no infinity
        assert not np.isinf(got[2])


def test_both_forms_are_close_in_the_middle(act):
    v = np.random.default_rng(2).standard_normal(50000).astype(np.float32)
    for fn in FNS:
        ref = reference(fn, v.astype(np.float64))
        rms = [float(np.sqrt(np.mean((act(e, fn, v) - ref) ** 2) / np.mean(ref ** 2))) for e in (True, False)]
        assert rms[0] < 6e-8 and rms[1] < 2e-7, (fn, rms)  # half a step of f32: at most 6e-8
