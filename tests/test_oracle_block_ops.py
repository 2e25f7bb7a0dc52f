"""The plain forms themselves: gradients against differences, the draws' statistics, the code table."""
import numpy as np
import pytest

from oracle import block_ops as ob
from oracle.select import splitmix64_stream

pytestmark = pytest.mark.cpu


def test_rotary_is_orthogonal_and_relative():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((1, 12, 2, 16))
    for nb in (False, True):
        y, _ = ob.rotary(x, None, [3, 4], [3, 4], nb)
        assert np.allclose((y * y).sum(-1), (x * x).sum(-1), atol=1e-12)
        assert np.allclose(ob.rotary(y, None, [3, 4], [3, 4], nb, inverse=True)[0], x, atol=1e-12)
        assert np.array_equal(y[..., 14:], x[..., 14:])
    # one token everywhere: inner products follow the distance alone
    q, k = np.broadcast_to(rng.standard_normal(16), (1, 12, 1, 16)), np.broadcast_to(rng.standard_normal(16), (1, 12, 1, 16))
    s = np.einsum("sd,td->st", ob.rotary(q, None, [3, 4], [4, 4])[0][0, :, 0], ob.rotary(k, None, [3, 4], [4, 4])[0][0, :, 0])
    assert np.allclose(s[0, 5], s[6, 11]) and np.allclose(s[1, 2], s[9, 10])


def test_draws_are_splitmix64_and_fair():
    seed, step = 77, 5
    keep = ob.drop_keep(50, 40, 0.25, seed, step)
    with np.errstate(over="ignore"):
        key = splitmix64_stream(int((np.uint64(seed) + np.uint64(step) * np.uint64(0x9E3779B97F4A7C15))), 1)[0]
    bits = splitmix64_stream(int(key), 500).view(np.uint16)        # little-endian: lowest bits first
    assert np.array_equal(keep, (bits >= 16384).reshape(50, 40))
    big = ob.drop_keep(1000, 1000, 0.1, 1, 2)
    assert abs(big.mean() - (1 - 6554 / 65536)) < 5 * np.sqrt(0.09 / 1e6)
    # pieces of a batch draw what the whole draws; rows of a group share
    assert np.array_equal(ob.drop_keep(20, 40, 0.25, seed, step, first_row=30), keep[30:])
    g = ob.drop_keep(12, 3, 0.5, 3, 4, group=4)
    assert (g == g[::4].repeat(4, 0)).all() and (g == g[:, :1]).all()
    assert ob.drop_keep(9, 9, 0.0, 1, 1).all() and not ob.drop_keep(9, 9, 1.0, 1, 1).any()
    assert ob.drop_factor(0.5) == 2.0 and ob.drop_factor(0.0) == 1.0 and ob.drop_factor(1.0) == 0.0


@pytest.mark.parametrize("rms,post,drop", [(False, True, False), (True, True, True), (False, False, True)])
def test_residual_norm_gradients_against_differences(rms, post, drop):
    rng = np.random.default_rng(3)
    B, S, D = 2, 3, 5
    x, y = rng.standard_normal((B, S, D)), rng.standard_normal((B, S, D))
    w = {k: rng.standard_normal(D) for k in ("post_w", "post_b", "res_scale", "pre_w", "pre_b")}
    w.update({k: rng.standard_normal((B, D)) for k in ("gate", "shift", "scale")})
    keep = rng.random((B, S, D)) > 0.3 if drop else None
    gx, gu = rng.standard_normal((B, S, D)), rng.standard_normal((B, S, D))

    def f():
        x1, u, k = ob.residual_norm(x, y, w, rms, post, 1e-3, keep, 1.4)
        return (x1 * gx).sum() + (u * gu).sum(), k

    dx, dy, g, _ = ob.residual_norm_bwd(f()[1], gx, gu)
    for t, d in [(x, dx), (y, dy)] + [(w[k], g[k]) for k in w if post or not k.startswith("post")]:
        for i in np.ndindex(*t.shape):
            t0 = t[i]
            t[i] = t0 + 1e-5
            a = f()[0]
            t[i] = t0 - 1e-5
            b = f()[0]
            t[i] = t0
            assert abs((a - b) / 2e-5 - d[i]) < 1e-6 * (1 + abs(d[i]))


def test_e4m3_codes():
    v = ob.e4m3_values()
    assert v[0x7E] == 448 and v[1] == 2.0 ** -9 and v[0x38] == 1.0 and np.isnan(v[0x7F])
    ok = ~np.isnan(v)
    assert np.array_equal(ob.e4m3_codes(v[ok]), np.arange(256)[ok].astype(np.uint8))
    # between neighbours: the nearer one, the even one from the middle
    for c in range(126):
        m = (v[c] + v[c + 1]) / 2
        assert ob.e4m3_codes(np.array([m]))[0] == (c if c % 2 == 0 else c + 1)
        assert ob.e4m3_codes(np.array([np.nextafter(m, 0)]))[0] == c
        assert ob.e4m3_codes(np.array([-np.nextafter(m, 500)]))[0] == c + 1 + 128


def test_f8_blocks():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((130, 200)) * np.exp(3 * rng.standard_normal((130, 1)))
    x[5] = 0
    x[7, 3] = np.inf
    for tile in (False, True):
        q, e, v = ob.f8_quantize(x, tile)
        assert q.shape == (130, 256) and e.shape == (2, 130) and (q[:, 200:][np.isfinite(v[:, -1])] & 0x7F == 0).all()
        with np.errstate(invalid="ignore"):
            err, top = np.abs(v - x), np.abs(x)
        good = np.isfinite(err)
        assert (err[good] <= np.maximum(top[good] / 16, 2.0 ** -10 * 2.0 ** (np.repeat(e.T.astype(int) - 127, 128, 1)[:, :200][good]))).all()
        assert np.isnan(v[7, :128]).all() and np.isfinite(v[7, 128:]).all()
    assert (ob.f8_quantize(x)[1][:, 5] == 1).all()
    for a, e in ((448.0, 0), (448.1, 1), (449.0 * 2.0 ** -20, -19), (1.75 * 2.0 ** 127, 119), (3e38, 119), (1e-45, -126)):
        assert ob.f8_quantize(np.array([[a, 0.0]]))[1][0, 0] == e + 127
