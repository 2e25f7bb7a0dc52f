"""The oracle of the eight-bit formats against hand-computed rows, the formats' own properties and
finite differences of the linear layer."""
import numpy as np
import pytest

from oracle import quant8 as oq

pytestmark = pytest.mark.cpu


def test_row_codes_by_hand():
    x = np.zeros((4, 64))
    x[0, :5] = [1.984375, -1.984375, 1.984375 / 2, 1.984375 / 254, 3 * 1.984375 / 254]   # ties 63.5, 0.5, 1.5
    x[1, :3] = [2.0, 1.0, -0.5]             # 127, 63.5, -31.75
    x[3, :2] = [np.inf, 1.0]
    q, s = oq.quant_rows(x)
    assert list(q[0, :5]) == [127, -127, 64, 0, 2]
    assert list(q[1, :3]) == [127, 64, -32]
    assert not q[2].any() and s[2] == 0
    assert not q[3].any() and np.isnan(s[3])
    assert s[0] == np.float32(1.984375) / np.float32(127)


def test_block_codes_by_hand():
    x = np.zeros((1, 128))
    x[0, :4] = [127.0, 0.5, 1.5, -2.5]       # e = 0: halves to even
    x[0, 32] = np.nextafter(127.0, 128.0)    # just above 127: e = 1
    x[0, 64] = np.nan
    q, e = oq.quant_blocks(x)
    assert list(q[0, :4]) == [127, 0, 2, -2] and e[0, 0] == 127
    assert q[0, 32] == 64 and e[0, 1] == 128
    assert e[0, 2] == 255 and not q[0, 64:96].any()
    assert e[0, 3] == 1
    v = oq.blocks_value(q, e)
    assert np.isnan(v[0, 64:96]).all() and np.isfinite(np.delete(v[0], np.s_[64:96])).all()


def test_errors_are_at_most_half_a_step():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((50, 256)) * np.exp(rng.standard_normal((50, 1)))).astype(np.float32).astype(np.float64)
    q, s = oq.quant_rows(x)
    a = np.abs(x).max(axis=1, keepdims=True)
    assert np.all(np.abs(q * a / 127 - x) <= a / 254 * (1 + 1e-12))
    q, e = oq.quant_blocks(x)
    step = np.repeat(2.0 ** (e.astype(np.float64) - 127), 32, axis=1)
    assert np.all(np.abs(oq.blocks_value(q, e) - x) <= step / 2)
    assert np.all(np.abs(q.reshape(50, -1, 32)).max(axis=2) >= 64)   # e is the smallest: the codes reach 64


def test_weight_gradient_equals_differences():
    rng = np.random.default_rng(5)
    M, N, K = 7, 8, 64
    q, e = oq.quant_blocks(rng.standard_normal((M, K)))
    xh = oq.blocks_value(q, e)
    W, b, dy = rng.standard_normal((N, K)), rng.standard_normal(N), rng.standard_normal((M, N))
    loss = lambda W, b: float((dy * np.tanh(0.0 * xh @ W.T + 1e-3 * (xh @ W.T + b)) * 1e3).sum())  # noqa: E731
    # the layer's output enters through a smooth function: dy' = dy (1 - tanh^2)
    t = np.tanh(1e-3 * (xh @ W.T + b))
    dw, db = oq.weight_grad(dy * (1 - t * t), q, e)
    V, u, h = rng.standard_normal((N, K)), rng.standard_normal(N), 1e-4
    num = (loss(W + h * V, b + h * u) - loss(W - h * V, b - h * u)) / (2 * h)
    ana = float((dw * V).sum() + (db * u).sum())
    assert abs(num - ana) <= 1e-7 * max(1.0, abs(ana))


@pytest.mark.parametrize("kind", ["preln", "adaln"])
def test_kept_backward_without_rounding_is_the_backward(kind, monkeypatch):
    # with a format that rounds nothing the kept backward is the block's own
    from oracle import block as oblk
    rng = np.random.default_rng(9)
    B, S, D, H, F = 2, 5, 64, 2, 128
    shapes = {"ln1_w": (D,), "ln1_b": (D,), "w_qkv": (3 * D, D), "b_qkv": (3 * D,), "w_o": (D, D), "b_o": (D,),
              "ln2_w": (D,), "ln2_b": (D,), "w_fc1": (F, D), "b_fc1": (F,), "w_fc2": (D, F), "b_fc2": (D,),
              "w_ada": (6 * D, D), "b_ada": (6 * D,)}
    p = {k: 0.2 * rng.standard_normal(s) + (1.0 if k in ("ln1_w", "ln2_w") else 0.0) for k, s in shapes.items()}
    cond = rng.standard_normal((B, D)) if kind == "adaln" else None
    h, dh = rng.standard_normal((B, S, D)), rng.standard_normal((B, S, D))
    _, cache = oblk.block_fwd(h, p, H, 1e-6, kind, cond)
    monkeypatch.setattr(oq, "kept", lambda t: t)
    got, want = oq.block_bwd_kept(dh, p, cache), oblk.block_bwd(dh, p, cache)
    np.testing.assert_allclose(got[0], want[0], rtol=1e-9, atol=1e-11)
    for k in p:
        np.testing.assert_allclose(got[1][k], want[1][k], rtol=1e-9, atol=1e-10)
    if kind == "adaln":
        np.testing.assert_allclose(got[2], want[2], rtol=1e-9, atol=1e-11)
