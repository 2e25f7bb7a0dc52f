"""Tensors of more than 2^31 elements: the last rows of one call equal a call on these rows alone, bit for bit."""
import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.gpu

TAIL = 5


def _filled(rows, cols, dtype):
    import torch
    x = torch.empty((rows, cols), dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    x[:1024] = torch.randn((1024, cols), generator=g, device="cuda").to(dtype)
    n = 1024
    while n < rows:   # the rows repeat
        k = min(n, rows - n)
        x[n:n + k] = x[:k]
        n += k
    return x


@pytest.mark.parametrize("N", [4096, 4099])
@pytest.mark.parametrize("group", [0, 2])
def test_dropout(N, group):
    import torch
    M = (1 << 31) // N + 1000
    x = _filled(M, N, torch.bfloat16)
    y = torch.empty_like(x)
    lo = (M - TAIL) // 8 * 8   # whole rows of 16 bytes for any N
    abi.sr_dropout(abi.SrDrop(p=0.3, seed=5, group=group), abi.SR_BF16, M, N, x, None, y)
    z = torch.empty_like(x[lo:])
    abi.sr_dropout(abi.SrDrop(p=0.3, seed=5, group=group, first_row=lo), abi.SR_BF16, M - lo, N, x[lo:], None, z)
    assert torch.equal(y[lo:], z)
    few = y[:4096]   # of a few rows all draws may be alike
    assert bool((few == 0).any()) and bool((few != 0).any())


@pytest.mark.parametrize("halves", [True, False])
def test_rotary(halves):
    import torch
    S, H, hd = (1 << 19) + 77, 32, 128   # 2^31 elements after 2^19 rows
    x = _filled(S, H * hd, torch.bfloat16)
    y = torch.empty_like(x)
    lay = abi.SR_ROT_HALVES if halves else abi.SR_ROT_NEIGHBOURS
    abi.sr_rotary(abi.SrRotary([S], [64], lay), 0, abi.SR_BF16, 1, S, H, hd, x, H * hd, None, 0, y, H * hd)
    z = torch.empty_like(x[-TAIL:])
    abi.sr_rotary(abi.SrRotary([S], [64], lay, origin=[float(S - TAIL)]), 0, abi.SR_BF16, 1, TAIL, H, hd, x[-TAIL:], H * hd, None, 0,
                  z, H * hd)
    assert torch.equal(y[-TAIL:], z)


@pytest.mark.parametrize("D", [4096, 1027])
def test_residual_norm(D):
    import torch
    S = (1 << 31) // D + 777
    x, y = _filled(S, D, torch.bfloat16), _filled(S, D, torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(4)
    w = {k: torch.randn(D, generator=g, device="cuda").bfloat16() for k in ("post_w", "post_b", "res_scale", "pre_w", "pre_b")}
    lo = (S - TAIL) // 8 * 8

    def run(x, y, first):
        cfg = abi.SrResidualNorm(B=1, S=x.shape[0], D=D, dtype=abi.SR_BF16, stream_dtype=abi.SR_BF16, norm=abi.SR_NORM_LAYER, post=1,
                                 eps=1e-6, mod_stride=0, drop=abi.SrDrop(p=0.2, seed=6, first_row=first))
        params = abi.residual_norm_params(**w)
        x1, u, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((4, x.shape[0]), device="cuda")
        abi.sr_residual_norm_fwd(cfg, params, x, y, x1, u, None, None, stats)
        grads = {k: torch.empty(D, device="cuda") for k in w}
        scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
        dx, dy = torch.empty_like(x), torch.empty_like(x)
        abi.sr_residual_norm_bwd(cfg, params, x1, y, stats, x, y, dx, dy, abi.residual_norm_grads(**grads), scratch)
        return x1, u, dx, dy, stats

    big = run(x, y, 0)
    part = run(x[lo:], y[lo:], lo)
    for a, b in zip(big[:4], part[:4]):
        assert torch.equal(a[lo:], b)
    assert torch.equal(big[4][:, lo:], part[4])


def test_quantize_f8():
    import torch
    M, N, ld = (1 << 15) + 40, 100, 1 << 16   # rows 2^16 elements apart: past 2^31 elements, a few of them read
    x = torch.zeros((M, ld), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    x[:, :N] = torch.randn((M, N), generator=g, device="cuda").bfloat16()
    far = abi.f8_buffers(M, N, transposed=True, rows=True)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_BF16, M, N, x, ld, *far)
    near = abi.f8_buffers(M, N, transposed=True, rows=True)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_BF16, M, N, x[:, :N].contiguous(), N, *near)
    assert torch.equal(far[0], near[0]) and torch.equal(far[2], near[2])
    assert torch.equal(far[1][:, :M], near[1][:, :M]) and torch.equal(far[3][:, :N], near[3][:, :N])


@pytest.mark.parametrize("M,N,K,act,dtype", [((1 << 20) - 3, 64, 2000, 0, "bf16"), (70, (1 << 20) - 3, 2000, 0, "bf16"),
                                             (32767, 32765, 129, 0, "bf16"), (32767, 32765, 129, 1, "bf16"),
                                             (64, 48, (1 << 24) - 5, 0, "f32"), (23169, 23169, 300, 0, "f32")])
def test_linear_f8(M, N, K, act, dtype):
    # codes and results just below 2 GiB, the longest rows; whole numbers up to 4, whose products and sums are exact in every order
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randint(-4, 5, (M, K), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    w = torch.randint(-4, 5, (N, K), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    xq, wq = abi.f8_buffers(M, K), abi.f8_buffers(N, K)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_BF16, M, K, x, K, *xq)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_BF16, N, K, w, K, *wq)
    dt, t = (abi.SR_BF16, torch.bfloat16) if dtype == "bf16" else (abi.SR_F32, torch.float32)
    y = torch.empty((M, N), dtype=t, device="cuda")
    scratch = torch.empty(max(abi.sr_linear_f8_scratch_bytes(M, N, K), 16), dtype=torch.uint8, device="cuda")
    abi.sr_linear_f8(dt, abi.SR_ACT_GELU if act else abi.SR_ACT_NONE, M, N, K, xq[0], xq[1], wq[0], wq[1], None, y, scratch)
    for rows, cols in ((slice(0, 20), slice(0, 20)), (slice(M - 20, M), slice(N - 20, N)), (slice(M - 20, M), slice(0, 20))):
        want = x[rows].double() @ w[cols].double().T
        if act:
            # half a step of bf16, and the activation's fit (5e-5 of z Phi(-|z|), which is 0.17 at most)
            want = torch.nn.functional.gelu(want)
            assert bool(((y[rows, cols].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all())
        else:
            assert torch.equal(y[rows, cols], want.to(t))
