"""The assembly scan for 64-bit shifts by an amount in a kernel's last vector register."""
import os

import pytest

from paper_2607_02829_amd import build
from paper_2607_02829_amd.isa_scan import high_shifts


def _kernel(ins, vgprs, name="_Zkernel"):
    return f"{name}:\n\t{ins}\n\ts_endpgm\n; NumVgprs: {vgprs}\n"


@pytest.mark.parametrize("ins,vgprs,bad", [
    ("v_lshrrev_b64 v[48:49], v55, v[48:49]", 56, True),
    ("v_lshlrev_b64 v[46:47], v55, v[46:47]", 56, True),
    ("v_ashrrev_i64 v[0:1], v7, v[2:3]", 8, True),
    ("v_lshl_add_u64 v[0:1], v[2:3], v15, v[4:5]", 16, True),
    ("v_lshrrev_b64 v[48:49], v55, v[48:49]", 57, False),   # the next register is there
    ("v_lshrrev_b64 v[48:49], v54, v[48:49]", 55, False),   # the last one used, not of the eight
    ("v_lshrrev_b64 v[48:49], 31, v[48:49]", 56, False),
    ("v_lshrrev_b64 v[48:49], s55, v[48:49]", 56, False),
    ("v_lshrrev_b32_e32 v48, v55, v48", 56, False),
])
def test_scan(ins, vgprs, bad):
    assert bool(high_shifts(_kernel(ins, vgprs))) == bad


def test_kernels_are_told_apart():
    asm = _kernel("v_lshrrev_b64 v[0:1], v7, v[2:3]", 9, "_Za") + _kernel("v_lshrrev_b64 v[0:1], v7, v[2:3]", 8, "_Zb")
    assert list(high_shifts(asm)) == ["_Zb"]


def test_built_kernels():
    if not all(os.path.exists(build.device_asm_path(s)) for s in build.ASYNC_READS | build.SHIFTS):
        pytest.skip("the kept assembly is made by a build here")
    assert build.check_shifts() == {}
