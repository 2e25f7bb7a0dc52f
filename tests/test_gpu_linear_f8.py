"""sr_quantize_f8 (codes and exponents exact) and sr_linear_f8 against their 64-bit forms.

Tolerances of a product over K, u = 2^-24, P = sum |x w|: fp32 results add exact products, eight or more to an instruction, so
at most K / 8 + 16 roundings of partial sums, (K / 8 + 16) u P; bf16 results come from instructions that drop, of eight products, what lies 2^-14
below the largest's leading bit, each product by less than 2^-13 of it: 7 x 2^-13 of the largest, so of P, at most; the typical size is pinned
apart.  Then bias (u) and half a step of the result's type."""
import numpy as np
import pytest

from oracle import block_ops as ob
from paper_2607_02829_amd import abi

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _sr(name):
    return abi.SR_BF16 if name == "bf16" else abi.SR_F32


def _same(got, want):
    """Equal codes; a zero's sign does not count for values, but it is kept: compare bytes."""
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]


@pytest.mark.parametrize("M,N", [(1, 1), (1, 128), (2, 3), (16, 129), (127, 128), (128, 127), (129, 300), (33, 1024), (257, 520)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", [False, True])
def test_codes(M, N, dtype, tile):
    import torch
    g = torch.Generator().manual_seed(M * 1000 + N)
    x = torch.randn((M, N), generator=g) * torch.exp(2 * torch.randn((M, 1), generator=g)) * torch.exp(torch.randn((1, N), generator=g))
    x = x.to(_dt(dtype))
    for extra, off in ((0, 0), (8, 0), (3, 1)):                     # strided rows, and rows off 16 bytes
        buf = torch.zeros(off + M * (N + extra) + 8, dtype=x.dtype)
        buf[off:off + M * (N + extra)].view(M, N + extra)[:, :N] = x
        xd = buf.cuda()[off:]
        bufs = abi.f8_buffers(M, N, True, True)
        for b in bufs:
            b.fill_(0xAB)
        abi.sr_quantize_f8(abi.SR_F8_TILE if tile else abi.SR_F8_ROW, _sr(dtype), M, N, xd, N + extra, *bufs)
        q, e, qt, et = (b.cpu().numpy() for b in bufs)
        x64 = x.double().numpy()
        wq, we, _ = ob.f8_quantize(x64, tile)
        _same(q, wq)
        _same(e[:, :M], we)
        wq, we, _ = ob.f8_quantize(x64.T, tile)
        _same(qt, wq)
        _same(et[:, :N], we)
        assert (e[:, M:] == 0xAB).all() and (et[:, N:] == 0xAB).all()
    only = abi.f8_buffers(M, N, False, True)
    abi.sr_quantize_f8(abi.SR_F8_TILE if tile else abi.SR_F8_ROW, _sr(dtype), M, N, x.cuda(), N, *only)
    assert np.array_equal(only[2].cpu().numpy(), qt)


def test_codes_at_the_borders():
    # ties between codes, values on both sides of an exponent's border, subnormals, the type's ends, zeros of both signs
    import torch
    v = ob.e4m3_values()[:127]
    rows = []
    for s in (1.0, 2.0 ** -126, 2.0 ** 100, 2.0 ** 119):
        mids = (v[:-1] + v[1:]) / 2
        r = np.concatenate([[448.0], mids, np.nextafter(mids.astype(np.float32), np.float32(0))])[:128].astype(np.float32)
        rows += [r * np.float32(s), -r * np.float32(s)]
    for top in (447.9, 448.0, 448.1, 449.0, 896.0, 897.0):
        rows.append(np.linspace(-top, top, 128).astype(np.float32))
    rows.append(np.full(128, 3.4e38, np.float32))
    rows.append(np.full(128, 1e-45, np.float32))
    rows.append(np.concatenate([np.zeros(64), -np.zeros(64)]).astype(np.float32))
    rows.append(np.concatenate([[1e-30], np.full(127, 1e-38)]).astype(np.float32))
    x = torch.from_numpy(np.stack(rows))
    q, e, qt, et = abi.f8_buffers(x.shape[0], 128, True, True)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_F32, x.shape[0], 128, x.cuda(), 128, q, e, qt, et)
    for got, ge, z in ((q, e, x), (qt, et, x.t())):
        wq, we, _ = ob.f8_quantize(z.double().numpy())
        _same(got.cpu().numpy(), wq)
        _same(ge.cpu().numpy()[:, :z.shape[0]], we)


def test_blocks_with_nan_and_inf():
    import torch
    x = torch.randn((140, 300), generator=torch.Generator().manual_seed(1))
    x[3, 5], x[70, 200], x[139, 299] = float("nan"), float("inf"), -float("inf")
    for tile in (False, True):
        bufs = abi.f8_buffers(140, 300, True, True)
        abi.sr_quantize_f8(int(tile), abi.SR_F32, 140, 300, x.cuda(), 300, *bufs)
        for q, e, z in ((bufs[0], bufs[1], x), (bufs[2], bufs[3], x.t())):
            _, we, wv = ob.f8_quantize(z.double().numpy(), tile)
            gv = ob.e4m3_values()[q.cpu().numpy()][:, :z.shape[1]]
            assert np.array_equal(np.isnan(gv), np.isnan(wv))
            assert np.array_equal(e.cpu().numpy()[:, :z.shape[0]], we)


def _codes(gen, R, C, spread=1.0):
    """Random values of codes and powers of two: what any quantiser may have written."""
    import torch
    v = torch.randn((R, C), generator=gen) * torch.exp(spread * torch.randn((R, 1), generator=gen))
    q, e, _, _ = abi.f8_buffers(R, C)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_F32, R, C, v.cuda(), C, q, e)
    qn, en = q.cpu().numpy(), e.cpu().numpy()[:, :R]
    vals = ob.e4m3_values()[qn] * 2.0 ** (np.repeat(en.T.astype(float), 128, 1) - 127)
    return q, e, vals[:, :C]


def _product(M, N, K, dtype, act=0, bias=True, spread=1.0, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed + M + 3 * N + 7 * K)
    xq, xe, xv = _codes(g, M, K, spread)
    wq, we, wv = _codes(g, N, K, spread)
    b = torch.randn(N, generator=g).to(_dt(dtype)) if bias else None
    y = torch.full((M * N + 32,), 7.25, dtype=_dt(dtype), device="cuda")
    n = abi.sr_linear_f8_scratch_bytes(M, N, K)
    scratch = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
    abi.sr_linear_f8(_sr(dtype), act, M, N, K, xq, xe, wq, we, None if b is None else b.cuda(), y,
                     None if scratch is None else scratch[:n])
    assert (y[M * N:] == 7.25).all() and (scratch is None or (scratch[n:] == 0xFF).all())
    got = y[:M * N].view(M, N)
    z = xv @ wv.T + (b.double().numpy() if bias else 0.0)
    P = np.abs(xv) @ np.abs(wv).T + (np.abs(b.double().numpy()) if bias else 0.0)
    return got, z, P


def _check(got, z, P, K, dtype, act=0):
    import torch
    got = got.cpu().double().numpy()
    assert np.isfinite(got).all()
    tol = P * (7 * 2.0 ** -13 if dtype == "bf16" else (K / 8 + 16) * U)
    want = z
    if act:   # the derivative of GELU is at most 1.13; its fit is good to 4e-7 of the value and 5e-5 of z Phi(-|z|)
        zt = torch.from_numpy(z)
        phi = torch.special.ndtr(-zt.abs()).numpy()
        want = z * torch.special.ndtr(zt).numpy()
        tol = 1.13 * tol + 4e-7 * np.abs(want) + 5e-5 * np.abs(z) * phi
    err = np.abs(got - want)
    tol = tol * (1 + 2.0 ** -7) + torch.finfo(_dt(dtype)).eps / 2 * np.abs(want) + 1e-37
    assert (err <= tol).all(), float((err / tol).max())
    # typical errors: a result's rounding is uniform (at most eps / 2 / sqrt 3 of it), and the dropped bits 4e-5 of the deviation of sums
    if z.size >= 64:
        rms = lambda t: float(np.sqrt(np.mean(np.square(t))))  # noqa: E731
        assert rms(err) <= torch.finfo(_dt(dtype)).eps / 2 / 3 ** 0.5 * rms(want) + (4e-5 if dtype == "bf16" else 4e-6) * rms(P)


SIZES = [(1, 1, 1), (1, 16, 128), (1, 4096, 1024), (3, 17, 129), (16, 64, 500), (5, 1024, 4096), (33, 276, 256), (64, 64, 64),
         (100, 130, 300), (128, 128, 128), (129, 257, 1000), (200, 1000, 70), (300, 300, 300), (257, 512, 640),
         (1000, 276, 256), (512, 1024, 1024), (2013, 1024, 256), (1030, 2050, 384), (4083, 276, 256), (4050, 1024, 512), (2111, 1023, 1030), (17000, 1030, 1024)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products(M, N, K, dtype):
    got, z, P = _product(M, N, K, dtype)
    _check(got, z, P, K, dtype)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 1024), (40, 100, 200), (300, 512, 256), (2000, 1024, 256), (129, 257, 130), (6500, 2100, 1024)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gelu_and_no_bias(M, N, K, dtype):
    got, z, P = _product(M, N, K, dtype, act=abi.SR_ACT_GELU, spread=0.2)
    _check(got, z, P, K, dtype, 1)
    got, z, P = _product(M, N, K, dtype, bias=False)
    _check(got, z, P, K, dtype)


@pytest.mark.parametrize("M,N,K", [(64, 64, 16200), (256, 128, 4096), (1024, 1024, 2013), (70, 300, 9000), (512, 512, 8192), (8, 24, 40000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_rows_with_few_results(M, N, K, dtype):
    # the weight gradient's shapes: sums cut into runs that are joined in a fixed order
    got, z, P = _product(M, N, K, dtype, bias=False)
    _check(got, z, P, K, dtype)
    again, _, _ = _product(M, N, K, dtype, bias=False)
    import torch
    assert torch.equal(got, again)


def test_far_powers_of_two():
    # exponents at both ends: products that fp32 holds, and ones that round to zero or infinity
    import torch
    M, N, K = 40, 48, 256
    for dtype in ("bf16", "f32"):
        for ex, ew in ((100, -95), (-100, 60), (-126, 119), (119, -126), (-40, -40), (50, 60)):
            g = torch.Generator().manual_seed(1)
            xv, wv = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g)
            xq, xe, _, _ = abi.f8_buffers(M, K)
            wq, we, _, _ = abi.f8_buffers(N, K)
            abi.sr_quantize_f8(0, abi.SR_F32, M, K, (xv * 2.0 ** -20).cuda(), K, xq, xe)
            abi.sr_quantize_f8(0, abi.SR_F32, N, K, (wv * 2.0 ** -20).cuda(), K, wq, we)
            xe.fill_(ex + 127)
            we.fill_(ew + 127)
            x64, w64 = (ob.e4m3_values()[q.cpu().numpy()] * 2.0 ** e for q, e in ((xq, ex), (wq, ew)))
            y = torch.empty((M, N), dtype=_dt(dtype), device="cuda")
            n = abi.sr_linear_f8_scratch_bytes(M, N, K)
            abi.sr_linear_f8(_sr(dtype), 0, M, N, K, xq, xe, wq, we, None, y, torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
            z, P = x64 @ w64.T, np.abs(x64) @ np.abs(w64).T
            with np.errstate(over="ignore"):
                err = np.abs(y.cpu().double().numpy() - z)
            # sums of magnitudes beyond the largest finite value may pass it on the way: an infinity is in order there
            over = P >= torch.finfo(_dt(dtype)).max
            assert over.any() == (ex + ew > 100)
            err[over & ~np.isfinite(err)] = 0
            tol = P * (7 * 2.0 ** -13 if dtype == "bf16" else (K / 8 + 16) * U) + torch.finfo(_dt(dtype)).eps / 2 * np.abs(z) + 2.0 ** -126
            assert (err <= tol).all(), (ex, ew)


def test_nan_blocks_reach_their_rows_only():
    import torch
    M, N, K = 200, 150, 400
    g = torch.Generator().manual_seed(4)
    x, w = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g)
    x[130, 390], w[20, 7] = float("nan"), float("inf")
    for dtype in ("bf16", "f32"):
        xq, xe, _, _ = abi.f8_buffers(M, K)
        wq, we, _, _ = abi.f8_buffers(N, K)
        abi.sr_quantize_f8(0, abi.SR_F32, M, K, x.cuda(), K, xq, xe)
        abi.sr_quantize_f8(0, abi.SR_F32, N, K, w.cuda(), K, wq, we)
        y = torch.empty((M, N), dtype=_dt(dtype), device="cuda")
        n = abi.sr_linear_f8_scratch_bytes(M, N, K)
        abi.sr_linear_f8(_sr(dtype), 0, M, N, K, xq, xe, wq, we, None, y, torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
        bad = torch.isnan(y).cpu()
        want = torch.zeros((M, N), dtype=torch.bool)
        want[130], want[:, 20] = True, True
        assert torch.equal(bad, want)


def test_the_three_products_of_a_layer():
    # y = x w^T, dx = dy w, dw = dy^T x on codes of one pass each, against products of the values
    import torch
    M, N, K = 333, 200, 260
    g = torch.Generator().manual_seed(6)
    x, w, dy = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g), torch.randn((M, N), generator=g).bfloat16()
    xb, wb, db = abi.f8_buffers(M, K, True, True), abi.f8_buffers(N, K, True, True), abi.f8_buffers(M, N, True, True)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_F32, M, K, x.cuda(), K, *xb)
    abi.sr_quantize_f8(abi.SR_F8_TILE, abi.SR_F32, N, K, w.cuda(), K, *wb)
    abi.sr_quantize_f8(abi.SR_F8_ROW, abi.SR_BF16, M, N, dy.cuda(), N, *db)
    rows = lambda t, tile=False: ob.f8_quantize(t.double().numpy(), tile)[2]  # noqa: E731
    xv, wv, dv = rows(x), rows(w, True), rows(dy)
    xc, dc = rows(x.t()).T, rows(dy.t()).T
    for (m, n, k), a, b, want, P in [((M, N, K), xb[:2], wb[:2], xv @ wv.T, np.abs(xv) @ np.abs(wv).T),
                                     ((M, K, N), db[:2], wb[2:], dv @ wv, np.abs(dv) @ np.abs(wv)),
                                     ((N, K, M), db[2:], xb[2:], dc.T @ xc, np.abs(dc.T) @ np.abs(xc))]:
        for dtype in ("bf16", "f32"):
            y = torch.empty((m, n), dtype=_dt(dtype), device="cuda")
            s = abi.sr_linear_f8_scratch_bytes(m, n, k)
            abi.sr_linear_f8(_sr(dtype), 0, m, n, k, *a, *b, None, y, torch.empty(max(s, 16), dtype=torch.uint8, device="cuda"))
            _check(y, want, P, k, dtype)
