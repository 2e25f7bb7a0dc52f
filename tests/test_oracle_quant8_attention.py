"""The oracle's backward of the kept values is that of a softmax: its probabilities sum to one, and it equals
differences of the attention of the kept q, k and v."""
import numpy as np
import pytest

from oracle import block as oblk
from oracle import quant8 as oq

pytestmark = pytest.mark.cpu


def _block(kind, logits, seed=3):
    rng = np.random.default_rng(seed)
    B, S, D, H, F = 2, 40, 64, 2, 128
    shapes = {"ln1_w": (D,), "ln1_b": (D,), "w_qkv": (3 * D, D), "b_qkv": (3 * D,), "w_o": (D, D), "b_o": (D,),
              "ln2_w": (D,), "ln2_b": (D,), "w_fc1": (F, D), "b_fc1": (F,), "w_fc2": (D, F), "b_fc2": (D,),
              "w_ada": (6 * D, D), "b_ada": (6 * D,)}
    p = {k: 0.15 * rng.standard_normal(s) + (1.0 if k in ("ln1_w", "ln2_w") else 0.0) for k, s in shapes.items()}
    cond = rng.standard_normal((B, D)) if kind == "adaln" else None
    h, dh = rng.standard_normal((B, S, D)), rng.standard_normal((B, S, D))
    _, c = oblk.block_fwd(h, p, H, 1e-6, kind, cond)
    f = np.sqrt(logits / (c["q"] @ c["k"].swapaxes(-1, -2) / np.sqrt(D // H)).std())
    p["w_qkv"][:2 * D] *= f
    p["b_qkv"][:2 * D] *= f
    return p, dh, oblk.block_fwd(h, p, H, 1e-6, kind, cond)[1], D, H


@pytest.mark.parametrize("logits", [1.0, 16.0, 64.0])
@pytest.mark.parametrize("kind", ["preln", "adaln"])
def test_probabilities_sum_to_one(kind, logits):
    p, dh, cache, D, _ = _block(kind, logits)
    _, g, _ = oq.block_bwd_kept(dh, p, cache)
    want = g["b_o"] @ p["w_o"]   # sum over keys of dv = sum over queries of dO
    assert np.linalg.norm(g["b_qkv"][2 * D:] - want) <= 1e-10 * np.linalg.norm(want)
    assert np.linalg.norm(g["b_qkv"][D:2 * D]) <= 1e-9 * np.linalg.norm(g["w_qkv"][D:2 * D])   # a shift of every key


@pytest.mark.parametrize("logits", [1.0, 16.0])
def test_kept_attention_equals_differences(logits, monkeypatch):
    p, dh, cache, D, H = _block("preln", logits)
    rec = []
    inner = oq._kept_attention_bwd
    monkeypatch.setattr(oq, "_kept_attention_bwd", lambda *a: rec.append((a, inner(*a))) or rec[-1][1])
    oq.block_bwd_kept(dh, p, cache)
    (args, grads), = rec
    x, dO = args[:3], args[-1]
    scale = 1.0 / np.sqrt(D // H)

    def f(q, k, v):
        s = q @ k.swapaxes(-1, -2) * scale
        e = np.exp(s - s.max(-1, keepdims=True))
        return float((dO * (e @ v / e.sum(-1, keepdims=True))).sum())

    rng = np.random.default_rng(4)
    for i in range(3):
        V, e = rng.standard_normal(x[i].shape), 1e-5
        up, down = (f(*(t + r * e * V if j == i else t for j, t in enumerate(x))) for r in (1, -1))
        num, ana = (up - down) / (2 * e), float((grads[i] * V).sum())
        # the third derivative's part e^2 / 6 x |s'|^3, |s'| the change of a logit along V (under 100), and rounding / e
        assert abs(num - ana) <= 1e-5 * np.sqrt(float((grads[i] ** 2).sum())) + 1e-6, (i, num, ana)
