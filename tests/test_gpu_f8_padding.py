"""Codes past a row's end are zeros, whatever its last block holds."""
import numpy as np
import pytest

from oracle import block_ops as ob
from paper_2607_02829_amd import abi

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N", [(1, 1), (3, 5), (140, 300), (129, 131), (70, 126), (257, 4), (17, 125)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", [False, True])
def test_quantize(M, N, bad, dtype, tile):
    import torch
    x = torch.randn((M, N), generator=torch.Generator().manual_seed(M + N))
    x[M - 1, N - 1] = x[M // 2, N - 1] = x[M - 1, 0] = bad
    x = x.bfloat16() if dtype == "bf16" else x
    bufs = abi.f8_buffers(M, N, True, True)
    for b in bufs:
        b.fill_(0x55)
    abi.sr_quantize_f8(int(tile), abi.SR_BF16 if dtype == "bf16" else abi.SR_F32, M, N, x.cuda(), N, *bufs)
    for q, e, z in ((bufs[0], bufs[1], x), (bufs[2], bufs[3], x.t())):
        wq, we, wv = ob.f8_quantize(z.double().numpy(), tile)
        q, n = q.cpu().numpy(), z.shape[1]
        assert (q[:, n:] == 0).all()
        gv = ob.e4m3_values()[q[:, :n]]
        assert np.array_equal(np.isnan(gv), np.isnan(wv)) and np.array_equal(q[:, :n][~np.isnan(wv)], wq[:, :n][~np.isnan(wv)])
        assert np.array_equal(e.cpu().numpy()[:, :z.shape[0]], we)


@pytest.mark.parametrize("D", [1, 2, 3, 5, 64, 126, 127, 130, 200, 255, 300, 1022, 1100, 2050])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_straight_from_the_norm(D, bad):
    import torch
    M = 9
    x = torch.randn((M, D), generator=torch.Generator().manual_seed(D))
    x[4, D - 1] = bad
    cfg = abi.SrResidualNorm(B=1, S=M, D=D, dtype=abi.SR_F32, stream_dtype=abi.SR_F32, norm=abi.SR_NORM_RMS, post=0, eps=1e-6, mod_stride=0)
    q, e, _, _ = abi.f8_buffers(M, D)
    q.fill_(0x55)
    abi.sr_residual_norm_fwd(cfg, abi.residual_norm_params(), x.cuda(), None, None, None, q, e)
    q = q.cpu().numpy()
    assert (q[:, D:] == 0).all()
    gv = ob.e4m3_values()[q[:, :D]]
    # a NaN takes the whole row with it; an infinity leaves its own block's codes NaN (Inf / Inf) and zeros elsewhere
    last = np.arange(D) // 128 == (D - 1) // 128
    assert np.isnan(gv[4]).all() if np.isnan(bad) else np.isnan(gv[4, last]).all() and (gv[4, ~last] == 0).all()
    assert np.isfinite(np.delete(gv, 4, 0)).all()
