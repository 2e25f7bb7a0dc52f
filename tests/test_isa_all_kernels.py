"""Every source with a kernel is among those whose assembly the build scans."""
import glob
import os

import pytest

from paper_2607_02829_amd import build

pytestmark = pytest.mark.cpu


def test_every_kernel_is_scanned():
    kernels = set()
    for path in glob.glob(os.path.join(build.CSRC, "*")):
        if path.endswith((".hip", ".cpp")):
            with open(path) as f:
                if "__global__" in f.read():
                    kernels.add(os.path.basename(path))
    assert kernels and kernels <= build.SHIFTS and build.SHIFTS <= set(build.SOURCES) and build.ASYNC_READS <= build.SHIFTS


def test_the_scan_sees_kernels_in_each():
    if not all(os.path.exists(build.device_asm_path(s)) for s in build.SHIFTS):
        pytest.skip("the kept assembly is made by a build here")
    for src in build.SHIFTS:
        with open(build.device_asm_path(src)) as f:
            text = f.read()
        if "amdhsa_kernel" not in text:   # templates of another source's kernels alone
            with open(os.path.join(build.CSRC, src)) as f:
                assert "__global__" not in f.read(), src
        else:
            assert "; NumVgprs:" in text, src
