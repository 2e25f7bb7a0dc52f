"""GELU of sr_linear8 in bf16: the exact one, rounded once."""
import numpy as np
import pytest

from oracle import quant8 as oq
from oracle.numerics import bf16_bits_to_f32, f32_to_bf16_bits, storage_to_f64
from paper_2607_02829_amd import abi, device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(16, 1024, 64), (300, 1024, 64), (1024, 512, 128), (4050, 1024, 64)])
def test_bf16_gelu_is_rounded_once(M, N, K):
    import torch
    print(f"[linear8 gelu] {M} x {N} x {K}", flush=True)
    rng = np.random.default_rng([M, N, K])
    xq = rng.integers(-127, 128, (M, K)).astype(np.int8)
    wq = rng.integers(-127, 128, (N, K)).astype(np.int8)
    # scales of powers of two and no bias: the pre-activation is exact in fp32 (a sum under 2^24), of deviation 1.3 (1.9)
    xs, ws = np.full(M, 2.0 ** -7, np.float32), np.full(N, 2.0 ** -8, np.float32)
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    abi.sr_linear8(abi.SR_BF16, abi.SR_ACT_GELU, M, N, K, device.to_device(xq), device.to_device(xs),
                   device.to_device(wq), device.to_device(ws), None, y)
    torch.cuda.synchronize()
    z = oq.linear(xq, xs, wq, ws)
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
