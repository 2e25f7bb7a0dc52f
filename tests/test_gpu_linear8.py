"""sr_linear8 against the fp64 oracle on the same codes and scales."""
import numpy as np
import pytest

from oracle import quant8 as oq
from oracle.numerics import storage_to_f64
from paper_2607_02829_amd import abi, device, inputs

pytestmark = pytest.mark.gpu

DT = {"bf16": abi.SR_BF16, "f32": abi.SR_F32}
GUARD = 64


def _data(M, N, K, dtype, seed=0, full=False):
    rng = np.random.default_rng([M, N, K, seed])
    lo, hi = (-127, 128) if not full else (126, 128)
    xq = rng.integers(lo, hi, (M, K)).astype(np.int8)
    wq = rng.integers(lo, hi, (N, K)).astype(np.int8)
    xs = np.exp(rng.standard_normal(M)).astype(np.float32) * np.float32(0.02)
    ws = np.exp(rng.standard_normal(N)).astype(np.float32) * np.float32(0.02 / 127)
    bias = inputs.to_storage(rng.standard_normal(N).astype(np.float32), dtype)
    return xq, xs, wq, ws, bias


def _run(M, N, K, dtype, data, act, use_bias):
    import torch
    xq, xs, wq, ws, bias = (device.to_device(a) for a in data)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((M * N + GUARD,), -9.0, dtype=dt, device="cuda")
    y = buf[:M * N].view(M, N)
    abi.sr_linear8(DT[dtype], act, M, N, K, xq, xs, wq, ws, bias if use_bias else None, y)
    torch.cuda.synchronize()
    assert bool((buf[M * N:] == -9.0).all())
    return device.to_host(y)


def _check(y, M, N, K, dtype, data, act, use_bias):
    xq, xs, wq, ws, bias = data
    b = storage_to_f64(bias) if use_bias else None
    v = oq.linear(xq, xs, wq, ws, b)
    want = oq.gelu(v) if act else v
    # fp32: the sum's rounding, two products, the bias: four half steps of the largest part
    part = np.abs(oq.linear(xq, xs, wq, ws)) + (np.abs(b)[None, :] if use_bias else 0.0)
    tol = 4 * 2.0 ** -24 * part
    if act:
        # |GELU'| <= 1.13 on the argument's error, and Phi's own: 2^-22 (fp32 activations) or 5e-5 (bf16) relative
        # to the smaller of Phi and 1 - Phi, and a part in 7e4 of the far negative tail (below -11.3 GELU is under 1e-28)
        tol = 1.13 * tol + (5e-5 if dtype == "bf16" else 1e-6) * np.abs(want) + 1.5e-5 * np.where(v < -4, np.abs(want), 0) + 1e-28
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    err = np.abs(storage_to_f64(y) - want)
    assert np.all(err <= tol), (float((err - tol).max()), np.argwhere(err > tol)[:4])


SHAPES = [
    (1, 8, 64), (1, 4096, 1024), (2, 1000, 192), (3, 64, 64), (5, 136, 320), (8, 256, 4096), (9, 40, 128),
    (16, 1024, 1024), (17, 72, 448), (31, 128, 64), (33, 200, 960), (64, 64, 64), (65, 64, 128), (100, 1032, 192),
    (128, 1024, 4096), (129, 264, 256), (257, 520, 576), (300, 16, 1024), (1000, 96, 2112),
]


@pytest.mark.parametrize("dtype,act,use_bias", [("bf16", 0, True), ("bf16", 1, True), ("f32", 1, True),
                                                 ("f32", 0, False)])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear_matches_oracle(M, N, K, dtype, act, use_bias):
    data = _data(M, N, K, dtype)
    _check(_run(M, N, K, dtype, data, act, use_bias), M, N, K, dtype, data, act, use_bias)


@pytest.mark.parametrize("M,N,K", [(4050, 1024, 1024), (4050, 4096, 1024), (2048, 1032, 4096), (8195, 2048, 256),
                                   (16200, 1024, 192)])
def test_linear_on_many_tokens(M, N, K):
    # fp64 on the GPU as the reference: sums of 127^2 K < 2^53 are exact there
    import torch
    data = _data(M, N, K, "bf16")
    xq, xs, wq, ws, bias = (device.to_device(a) for a in data)
    for act in (0, 1):
        y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        abi.sr_linear8(abi.SR_BF16, act, M, N, K, xq, xs, wq, ws, bias, y)
        v = (xq.double() @ wq.double().t().contiguous()) * xs.double()[:, None] * ws.double()[None, :]
        part = v.abs() + bias.double().abs()[None, :]
        v = v + bias.double()[None, :]
        want = 0.5 * v * torch.erfc(v * -(0.5 ** 0.5)) if act else v
        tol = (1.13 * 4 * 2.0 ** -24 * part + (7e-5 if act else 0.0) * want.abs() + 1e-28) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
        assert bool(((y.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype,act", [("bf16", 0), ("bf16", 1), ("f32", 0), ("f32", 1)])
@pytest.mark.parametrize("M,N,K", [
    # sizes on either side of every border between tile shapes, ragged in rows, columns and the last 64 of k
    (600, 600, 192), (600, 600, 576), (500, 1032, 2112), (1500, 1032, 448), (2050, 1032, 2112), (4050, 1000, 320),
    (4100, 3336, 1088), (3600, 3600, 2112), (3500, 4104, 64), (8200, 4104, 192), (2040, 64, 64), (2064, 64, 64), (250, 250 * 8, 1024),
])
def test_linear_on_every_tile_shape(M, N, K, dtype, act):
    data = _data(M, N, K, dtype, seed=1)
    _check(_run(M, N, K, dtype, data, act, True), M, N, K, dtype, data, act, True)


@pytest.mark.parametrize("M,N,K", [(1 << 20, 8, 64), (1, 1 << 18, 64), (3, 1 << 17, 128), (30011, 24, 65536 // 2)])
def test_linear_at_extreme_shapes(M, N, K):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(K)
    xq = torch.randint(-127, 128, (M, K), generator=gen, device="cuda", dtype=torch.int8)
    wq = torch.randint(-127, 128, (N, K), generator=gen, device="cuda", dtype=torch.int8)
    xs, ws = torch.rand(M, generator=gen, device="cuda"), torch.rand(N, generator=gen, device="cuda")
    y = torch.empty((M, N), device="cuda")
    abi.sr_linear8(abi.SR_F32, 0, M, N, K, xq, xs, wq, ws, None, y)
    for lo in range(0, M, 1 << 14):   # sums in fp64 by rows: exact
        acc = xq[lo:lo + (1 << 14)].double() @ wq.double().t().contiguous()
        want = acc.float() * xs[lo:lo + (1 << 14), None] * ws[None, :]
        assert torch.equal(y[lo:lo + (1 << 14)], want)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_largest_sums_are_exact(M):
    # codes of 126 and 127 over the longest K: sums near 2^30, beyond what fp32 holds exactly
    N, K = 24, 65536
    data = _data(M, N, K, "f32", full=True)
    y = _run(M, N, K, "f32", data, 0, False)
    xq, xs, wq, ws, _ = data
    acc = xq.astype(np.int64) @ wq.astype(np.int64).T
    want = (acc.astype(np.float32) * xs[:, None]).astype(np.float32) * ws[None, :]
    assert np.array_equal(y, want.astype(np.float32))


def test_extreme_codes():
    # -128 is no code of the quantiser but a legal operand
    M, N, K = 33, 40, 128
    xq, xs, wq, ws, bias = _data(M, N, K, "f32")
    xq[:] = -128
    wq[:20] = -128
    data = (xq, xs, wq, ws, bias)
    _check(_run(M, N, K, "f32", data, 0, True), M, N, K, "f32", data, 0, True)


@pytest.mark.parametrize("M", [2, 70])
def test_a_non_finite_token_stays_alone(M):
    N, K = 64, 128
    xq, xs, wq, ws, bias = _data(M, N, K, "bf16")
    clean = _run(M, N, K, "bf16", (xq, xs, wq, ws, bias), 1, True)
    xs2, xq2 = xs.copy(), xq.copy()
    xs2[1], xq2[1] = np.nan, 0
    y = _run(M, N, K, "bf16", (xq2, xs2, wq, ws, bias), 1, True)
    assert np.isnan(storage_to_f64(y)[1]).all()
    keep = np.arange(M) != 1
    assert np.array_equal(y[keep], clean[keep])


@pytest.mark.parametrize("M,K", [(1, 64), (40, 256), (3, 1024)])
def test_zero_tokens_give_the_bias(M, K):
    N = 72
    xq, xs, wq, ws, bias = _data(M, N, K, "f32")
    xq[0], xs[0] = 0, 0.0
    y = _run(M, N, K, "f32", (xq, xs, wq, ws, bias), 0, True)
    assert np.array_equal(y[0], storage_to_f64(bias).astype(np.float32))


def test_a_token_does_not_depend_on_its_batch():
    # integer sums: whatever shape the batch selects, a token's bits are the same
    N, K = 200, 320
    xq, xs, wq, ws, bias = _data(700, N, K, "f32")
    whole = _run(700, N, K, "f32", (xq, xs, wq, ws, bias), 1, True)
    for lo, n in ((0, 1), (3, 7), (100, 33), (320, 130), (650, 50)):
        part = _run(n, N, K, "f32", (xq[lo:lo + n], xs[lo:lo + n], wq, ws, bias), 1, True)
        assert np.array_equal(part, whole[lo:lo + n]), (lo, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(2, 64, 128), (130, 72, 576), (600, 600, 192), (2100, 1032, 192), (4100, 3336, 1088)])
def test_infinite_pre_activations(M, N, K, dtype):
    # GELU(+Inf) = +Inf and GELU(-Inf) = 0, from an infinite bias and from scales whose product overflows
    data = list(_data(M, N, K, dtype))
    bias = storage_to_f64(data[4]).astype(np.float32)
    bias[1], bias[N - 2] = np.inf, -np.inf
    data[4] = inputs.to_storage(bias, dtype)
    data[1], data[3] = data[1].copy(), data[3].copy()
    data[1][0], data[3][2] = 1e25, 1e20
    data[0][0], data[2][2], data[2][N - 3] = 100, 100, -100   # sums of one sign in row 0
    data[3][N - 3] = 1e20
    clean = [1, 2, N - 3, N - 2]
    for act in (0, 1):
        y = storage_to_f64(_run(M, N, K, dtype, tuple(data), act, True))
        low = 0.0 if act else -np.inf
        assert (y[:, 1] == np.inf).all() and (y[:, N - 2] == low).all()
        assert y[0, 2] == np.inf and y[0, N - 3] == low
        assert np.isfinite(np.delete(y[1:], clean, axis=1)).all()


@pytest.mark.parametrize("dtype,act", [("bf16", 0), ("bf16", 1), ("f32", 1)])
@pytest.mark.parametrize("M,N,K", [(1, 1024, 4096), (16, 4096, 4096), (17, 2040, 2112), (64, 1024, 8192), (70, 808, 4160),
                                   (256, 256, 4096), (60, 8, 65536)])
def test_linear_on_few_tokens_of_long_rows(M, N, K, dtype, act):
    data = _data(M, N, K, dtype, seed=2)
    _check(_run(M, N, K, dtype, data, act, True), M, N, K, dtype, data, act, True)
