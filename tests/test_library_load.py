"""One HIP runtime in a process, whichever of the library and PyTorch a program turns to first."""
import os
import subprocess
import sys

import pytest

from paper_2301_01333_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
from paper_2301_01333_amd import binding
binding.lib()
import torch
print(len({line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line}))
"""


@pytest.mark.skipif(not os.path.exists(binding.LIB_PATH), reason="libogc_mlp.so not built (python -m paper_2301_01333_amd.build)")
def test_the_library_before_pytorch():
    pytest.importorskip("torch")
    out = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert (out.returncode, out.stdout.strip()) == (0, "1"), out.stdout + out.stderr
