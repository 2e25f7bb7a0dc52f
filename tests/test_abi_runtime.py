"""One HIP runtime per process, whichever of libsr and torch is asked for first."""
import subprocess
import sys

import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.cpu

CODE = """
import ctypes
from paper_2607_02829_amd import abi
n = ctypes.c_size_t()
abi.lib().sr_weight_grad8_scratch_bytes(abi.SR_BF16, 100, 64, 64, ctypes.byref(n))
import torch
print(len({l.split()[-1] for l in open("/proc/self/maps") if "libamdhip64" in l}))
"""


def test_the_library_before_torch():
    try:
        abi.lib()
    except abi.SrLibraryMissing as e:
        pytest.skip(str(e))
    r = subprocess.run([sys.executable, "-c", CODE], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-500:]
    assert r.stdout.strip() == "1"
