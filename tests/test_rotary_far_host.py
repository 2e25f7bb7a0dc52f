"""sr_rotary refuses angles that 64 bits cannot hold to a useful fraction of a turn: more than 2^45 anywhere on the grid."""
import ctypes

import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.cpu

FAKE = 1 << 40          # aligned, never dereferenced: validation fails first
FAR = 2.0 ** 45


def _call(S=8, x=FAKE, **kw):
    try:
        lib = abi.lib()
    except abi.SrLibraryMissing as e:
        pytest.skip(str(e))
    rot = abi.SrRotary(**kw)
    return lib.sr_rotary(ctypes.byref(rot), 0, abi.SR_F32, 1, S, 2, 16, x, 32, None, 0, FAKE + 4096, 32, None)


@pytest.mark.parametrize("kw", [
    dict(grid=[8], pairs=[4], origin=[FAR + 1]), dict(grid=[8], pairs=[4], origin=[-FAR - 1]),
    dict(grid=[8], pairs=[4], origin=[1.7e18]),                                 # nanoseconds
    dict(grid=[8], pairs=[4], origin=[1e300], step=[1e300]),
    dict(grid=[8], pairs=[4], origin=[1.7e308], step=[1.7e308]),                # places beyond the type
    dict(grid=[8], pairs=[4], origin=[FAR - 6]),                                # the last place alone
    dict(grid=[8], pairs=[4], origin=[FAR], step=[1.0]), dict(grid=[8], pairs=[4], step=[-FAR / 6]),
    dict(grid=[2, 8], pairs=[2, 3], origin=[0.0, 3e10], freqs=[1.0, 1.0, 1.0, 0.5, -1173.0]),
    dict(grid=[8], pairs=[4], origin=[1.0], base=1e-300),                       # frequencies up to 10^225
])
def test_far_angles_are_refused(kw):
    assert _call(**kw) == abi.SR_EUNSUPPORTED
    assert b"2^45" in abi.lib().sr_last_error()
