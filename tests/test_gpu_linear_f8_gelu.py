"""GELU of sr_linear_f8 in bf16: the exact one of the sum, rounded once."""
import numpy as np
import pytest

from oracle import block_ops as ob
from oracle import quant8 as oq
from oracle.numerics import bf16_bits_to_f32, f32_to_bf16_bits, storage_to_f64
from paper_2607_02829_amd import abi, device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(16, 1024, 64), (300, 1024, 100), (256, 512, 512), (512, 1024, 700), (1024, 1024, 300), (2013, 1024, 256),
                                   (4050, 1024, 512), (4083, 1030, 200), (8100, 1024, 1024), (16200, 1024, 1024), (64, 512, 6000)])
def test_bf16_gelu_is_rounded_once(M, N, K):
    import torch
    print(f"[linear_f8 gelu] {M} x {N} x {K}", flush=True)
    rng = np.random.default_rng([M, N, K])
    x, w = rng.integers(-7, 8, (M, K)).astype(np.float64), rng.integers(-7, 8, (N, K)).astype(np.float64)
    # whole numbers under 8, whose products and sums are exact in every order (under 2^24, and a product of 1 lies less than 2^6 below the
    # largest), times a power of two that gives pre-activations of deviation 1 to 2 (18.7 K^(1/2) before it); a bias of whole units
    unit = -int(np.floor(np.log2(18.7 * K ** 0.5)))
    bias = rng.integers(-30, 31, N)
    xq, xe, _, _ = abi.f8_buffers(M, K)
    wq, we, _, _ = abi.f8_buffers(N, K)
    for v, q, e in ((x, xq, xe), (w, wq, we)):
        codes = np.zeros(q.shape, np.uint8)
        codes[:, :K] = ob.e4m3_codes(v)
        q.copy_(torch.from_numpy(codes))
    xe.fill_(127)
    we.fill_(127 + unit)
    b = torch.from_numpy(bias * 2.0 ** unit).bfloat16().cuda()
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(max(abi.sr_linear_f8_scratch_bytes(M, N, K), 16), dtype=torch.uint8, device="cuda")
    abi.sr_linear_f8(abi.SR_BF16, abi.SR_ACT_GELU, M, N, K, xq, xe, wq, we, b, y, scratch)
    torch.cuda.synchronize()
    z = (x @ w.T + bias) * 2.0 ** unit
    near = np.abs(z) <= 4.0
    want = oq.gelu(z)
    got = storage_to_f64(device.to_host(y))
    # In fp32 Phi(-|z|) = t 2^(q - z^2 log2(e) / 2): the fit within 2e-7, an exponent under 16 (half a step of it is
    # 2^-21, times log 2), a reciprocal and a power within a step, four roundings of 2^-24:  2e-7 + 3.3e-7 + 2.4e-7 +
    # 2.4e-7 = 1.0e-6 of the value.  A bf16 result is another than the rounded exact one only within that of a border
    # between two, and borders lie at least 2^-8 of the value apart: a share of at most 2 x 1.0e-6 x 2^8 = 5.2e-4.
    other = (got != bf16_bits_to_f32(f32_to_bf16_bits(want))) & near
    assert other.sum() <= 5.2e-4 * near.sum(), float(other.sum() / near.sum())
    assert np.all((np.abs(got - want) <= (2.0 ** -8 + 1.1e-6) * np.abs(want) + 1e-38) | ~near)
