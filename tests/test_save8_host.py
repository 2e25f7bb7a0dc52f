"""Workspace sizes of SR_BLOCK_SAVE8 for any number of blocks: no memory is taken to say them."""
import subprocess
import sys

import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.cpu

CODE = """
import resource
from paper_2607_02829_amd import abi
abi.lib()
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (1 << 28), used + (1 << 28)))
def saved(n):
    cfg = abi.SrConfig(B=1, L=10, D=64, H=2, F=128, n_blocks=n, dtype=abi.SR_BF16, kind=KIND | abi.SR_BLOCK_SAVE8, ln_eps=1e-6,
                       idx_shared=0)
    return abi.sr_workspace_bytes(cfg, 10)[0]
n = 5_000_000
assert saved(n) == saved(1) + (n - 1) * (saved(2) - saved(1))
"""


@pytest.mark.parametrize("kind", [abi.SR_BLOCK_PRELN, abi.SR_BLOCK_ADALN])
def test_many_blocks(kind):
    try:
        abi.lib()
    except abi.SrLibraryMissing as e:
        pytest.skip(str(e))
    r = subprocess.run([sys.executable, "-c", CODE.replace("KIND", str(kind))], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-500:]
