"""The plain codes of a block with an Inf or NaN: NaN for its values, zeros past the row's end."""
import numpy as np
import pytest

from oracle import block_ops as ob

pytestmark = pytest.mark.cpu


@pytest.mark.parametrize("tile", [False, True])
def test_padding_of_nan_blocks(tile):
    x = np.random.default_rng(2).standard_normal((5, 130))
    x[1, 129], x[3, 128] = np.nan, np.inf
    q, e, v = ob.f8_quantize(x, tile)
    assert q.shape == (5, 256) and (q[:, 130:] == 0).all()
    rows = np.ones(5, bool) if tile else np.isin(np.arange(5), (1, 3))
    assert np.isnan(v[rows, 128:]).all() and (q[rows, 128:130] == 0x7F).all() and np.isfinite(v[~rows]).all() and (e[1, rows] == 127).all()
