"""sr_linear_f8 on blocks of the lowest exponents: fp32 results take their values in bf16, whose last bit is 2^-133."""
import numpy as np
import pytest

from oracle import block_ops as ob
from paper_2607_02829_amd import abi

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(16, 128, 128), (130, 128, 600), (512, 512, 512), (300, 2000, 256), (1030, 1030, 1024), (64, 128, 6000)])
@pytest.mark.parametrize("e", [-126, -125, -124, -123, -117])
@pytest.mark.parametrize("weights", [False, True])
def test_values_of_low_blocks(M, N, K, e, weights):
    # one operand's rows hold every finite code, the other's a single one of 2^119: a result is one value, raised by 2^119
    import torch
    codes = np.concatenate([np.arange(127), [0x80 + 5]]).astype(np.uint8)

    def operand(rows, ones):
        q, ex, _, _ = abi.f8_buffers(rows, K)
        t = np.zeros(q.shape, np.uint8)
        if ones:
            t[np.arange(rows), np.arange(rows) % 128] = 0x38
        else:
            t[:, :128] = codes
        q.copy_(torch.from_numpy(t))
        ex.fill_((119 if ones else e) + 127)
        return q, ex

    x, w = operand(M, weights), operand(N, not weights)
    value = ob.e4m3_values()[codes] * 2.0 ** e
    for dtype, t in ((abi.SR_F32, torch.float32), (abi.SR_BF16, torch.bfloat16)):
        y = torch.empty((M, N), dtype=t, device="cuda")
        scratch = torch.empty(max(abi.sr_linear_f8_scratch_bytes(M, N, K), 16), dtype=torch.uint8, device="cuda")
        abi.sr_linear_f8(dtype, abi.SR_ACT_NONE, M, N, K, *x, *w, None, y, scratch)
        got = y.cpu().double().numpy() * 2.0 ** -119
        want = np.rint(value * 2.0 ** 133) * 2.0 ** -133 if dtype == abi.SR_F32 else value   # rint: halves to the even one
        want = np.broadcast_to(want[np.arange(N) % 128], (M, N)) if not weights else np.broadcast_to(want[np.arange(M) % 128][:, None], (M, N))
        assert np.array_equal(got, want)
