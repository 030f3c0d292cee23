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


def test_every_name_is_there():
    """The names that the package's functions look up among their module's, or the builtins."""
    import builtins
    import dis
    import importlib
    import types

    def names(code):
        for i in dis.get_instructions(code):
            if i.opname in ("LOAD_GLOBAL", "LOAD_NAME"):
                yield i.argval
        for c in code.co_consts:
            if isinstance(c, types.CodeType):
                yield from names(c)

    for module in ("_lib", "context", "ops", "ops4", "sched"):
        m = importlib.import_module("paper_2505_08944_amd." + module)
        for f in vars(m).values():
            for g in (vars(f).values() if isinstance(f, type) and f.__module__ == m.__name__ else (f,)):
                if isinstance(g, types.FunctionType) and g.__module__ == m.__name__:
                    for name in names(g.__code__):
                        assert hasattr(m, name) or hasattr(builtins, name), (module, g.__qualname__, name)
