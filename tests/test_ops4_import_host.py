"""CPU: the package asks nothing of torch that only newer versions have."""

import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_torch_without_types_of_4_bits():
    code = ("import torch\n"
            "for name in ('float4_e2m1fn_x2', 'float8_e8m0fnu'):\n"
            "    if hasattr(torch, name): delattr(torch, name)\n"
            "import paper_2505_08944_amd as aep\n"
            "assert aep.Linear and aep.Linear4 and aep.Cache4\n"
            "for call in (lambda: aep.quantize_mx4(torch.zeros(2, 32)),\n"
            "             lambda: aep.dequantize_mx4(torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(2, 1, dtype=torch.uint8), 32)):\n"
            "    try: call()\n"
            "    except ValueError: continue\n"
            "    raise AssertionError('not refused')\n")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT)
