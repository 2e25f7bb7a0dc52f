"""Scratch sizes of the residual step's backward and of products on 8-bit codes never fall with a larger call, so that the scratch
of the largest one serves them all."""
import random

import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.cpu


@pytest.fixture(autouse=True)
def _library():
    try:
        abi.lib()
    except abi.SrLibraryMissing as e:
        pytest.skip(str(e))


def _norm(B, S, D):
    return abi.sr_residual_norm_scratch_bytes(abi.SrResidualNorm(B=B, S=S, D=D, dtype=abi.SR_BF16, stream_dtype=abi.SR_F32, norm=abi.SR_NORM_RMS,
                                                                 post=1, eps=1e-6, mod_stride=D))


def _log(rng, hi):
    return int(round(hi ** rng.random()))


@pytest.mark.parametrize("D", [1, 64, 128, 129, 256, 257, 512, 1000, 1024, 1025, 2048, 2049, 4096, 4097, 8192])
@pytest.mark.parametrize("B", [1, 3, 8, 255, 256, 257, 600])
def test_residual_norm_by_rows(B, D):
    last = 0
    for S in [*range(1, 40), *range(250, 262), 511, 512, 513, 1024, 1025, 2047, 2048, 2049, 4097, 16200, 10 ** 5, 3 * 10 ** 6]:
        n = _norm(B, S, D)
        assert n >= last, (S, n, last)
        last = n
    assert last <= max(1023, B) * 16 * D


def test_residual_norm_by_all_sizes():
    rng = random.Random(3)
    for _ in range(3000):
        B, S, D = _log(rng, 1 << 12), _log(rng, 1 << 18), _log(rng, 8192)
        assert _norm(B, S, D) >= _norm(rng.randint(1, B), rng.randint(1, S), rng.randint(1, D))


@pytest.mark.parametrize("N,K", [(64, 16384), (256, 4096), (1024, 16200), (64, 5120), (1, 1 << 20)])
def test_linear_f8_by_tokens(N, K):
    last = 0
    for M in [*range(1, 40), 64, 127, 128, 129, 256, 511, 1024, 1025, 2048, 4097, 5000, 16200, 16500]:
        if M * (K + 127) >= 1 << 31:
            break
        n = abi.sr_linear_f8_scratch_bytes(M, N, K)
        assert n >= last, (M, n, last)
        last = n


def test_linear_f8_by_all_sizes():
    rng = random.Random(4)
    for _ in range(5000):
        M, N, K = _log(rng, 1 << 15), _log(rng, 1 << 13), _log(rng, 1 << 15)
        assert abi.sr_linear_f8_scratch_bytes(M, N, K) >= abi.sr_linear_f8_scratch_bytes(rng.randint(1, M), rng.randint(1, N), rng.randint(1, K))
    assert abi.sr_linear_f8_scratch_bytes(16200, 4096, 4096) == 0   # short rows need none
