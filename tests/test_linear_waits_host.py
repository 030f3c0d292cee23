"""Wait states around the tiled product's direct-to-LDS loads, in the built
code: the same reading of it as for the FFN's (test_ffn_waits_host.py)."""

import os
import subprocess

import pytest

from paper_2505_08944_amd import build
from test_ffn_waits_host import _kernels, _too_close


def test_loads_wait_for_their_scalar_registers(tmp_path):
    try:
        cc = build.hipcc()
    except RuntimeError:
        pytest.skip("needs hipcc")
    out = str(tmp_path / "k_linear_tiles.s")
    flags = [f for f in build.CFLAGS if f not in ("-fPIC",)]
    subprocess.run([cc, *flags, "-w", "-S", "--cuda-device-only", os.path.join(build.CSRC, "k_linear_tiles.hip"), "-o",
                    out], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    kernels = {n: b for n, b in _kernels(open(out).read()).items() if "linear_tiles_kernel" in n}
    assert len(kernels) == 2
    for name, blocks in kernels.items():
        loads, bad = _too_close(blocks)
        assert loads > 30, name
        assert not bad, (name, bad[:4])
