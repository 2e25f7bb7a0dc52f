"""Eight-bit activations in fp64: the two code formats, the linear layer on codes, and the weight
gradient from a checkpoint.  Plain formulas, no code shared with the GPU path.

Row format: q = 127 x / max|x| to the nearest integer (halves to even), value q * fl32(max|x| / 127).
Block format: 2^e per 32 channels, e the smallest integer in [-126, 121] with max|x| <= 127 2^e,
q = x 2^-e to the nearest integer within +-127, value q 2^e."""
from __future__ import annotations

import numpy as np
from scipy.special import erfc

from . import block as blk

BLOCK = 32


def quant_rows(x):
    """x (M, N) fp64 holding fp32 (or bf16) values -> codes int8 (M, N), scales fp32 (M,)."""
    x = np.asarray(x, np.float64)
    a = np.abs(x).max(axis=1)
    bad = ~np.isfinite(x).all(axis=1)
    safe = np.where((a > 0) & ~bad, a, 1.0)
    # 127 x is exact; the quotient of a 31-bit and a 24-bit integer cannot round onto a half it is not
    q = np.rint(127.0 * np.where(bad[:, None], 0.0, x) / safe[:, None]).astype(np.int8)
    scale = np.where(bad, np.float32(np.nan), (np.where(bad, 0.0, a).astype(np.float32) / np.float32(127.0)))
    return q, scale.astype(np.float32)


def rows_value(q, scale):
    return q.astype(np.float64) * scale.astype(np.float64)[:, None]


def quant_blocks(x):
    """x (M, N) fp64 -> codes int8 (M, N), exponent bytes uint8 (M, N / 32)."""
    x = np.asarray(x, np.float64)
    b = x.reshape(x.shape[0], -1, BLOCK)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[..., None], 0.0, b)
    a = np.abs(b).max(axis=2)
    e = np.full(a.shape, -126, np.int64)
    for k in range(-126, 121):   # the first exponent whose 127 2^e reaches the maximum
        e = np.where((e == k) & (a > 127.0 * 2.0 ** k), k + 1, e)
    q = np.clip(np.rint(b * 2.0 ** -e[..., None].astype(np.float64)), -127, 127).astype(np.int8)
    return q.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def blocks_value(q, eb):
    s = np.where(eb == 255, np.nan, 2.0 ** (eb.astype(np.float64) - 127.0))
    return (q.reshape(q.shape[0], -1, BLOCK) * s[..., None]).reshape(q.shape)


def gelu(v):
    return 0.5 * v * erfc(-v / np.sqrt(2.0))


def linear(xq, xs, wq, ws, bias=None, act_gelu=False):
    """y (M, N) fp64 = act(xs ws (xq wq^T) + bias)."""
    v = (xq.astype(np.float64) @ wq.astype(np.float64).T) * xs.astype(np.float64)[:, None] * ws.astype(np.float64)[None, :]
    if bias is not None:
        v = v + bias[None, :]
    return gelu(v) if act_gelu else v


def weight_grad(dy, q, eb):
    """dw (N, K), db (N,) fp64 from dy (M, N) and the block-format checkpoint of the layer's input."""
    dy = np.asarray(dy, np.float64)
    return dy.T @ blocks_value(q, eb), dy.sum(axis=0)


def kept(t):
    """The values that an activation (..., channels) has after being kept in the block format."""
    t2 = t.reshape(-1, t.shape[-1])
    return blocks_value(*quant_blocks(t2)).reshape(t.shape)


def _kept_attention_bwd(q, k, v, dO):
    """dq, dk, dv (B, H, S, hd) of the attention of the kept q, k and v: its probabilities and output, not the
    forward's, so that the rows of P sum to one and those of dS to zero."""
    scale = 1.0 / np.sqrt(q.shape[-1])
    s = q @ k.swapaxes(-1, -2) * scale
    P = np.exp(s - s.max(-1, keepdims=True))
    P /= P.sum(-1, keepdims=True)
    dS = P * (dO @ v.swapaxes(-1, -2) - (dO * (P @ v)).sum(-1, keepdims=True))
    return dS @ k * scale, dS.swapaxes(-1, -2) @ q * scale, P.swapaxes(-1, -2) @ dO


def _shift(cache, n):
    """The adaLN shift (B, 1, D) of LayerNorm n, from its output u = n (1 + scale) + shift."""
    u, x = cache["u" if n == "1" else "u2"], cache["n" + n]
    return (u - x * (1.0 + cache["sc" + n])).mean(axis=1, keepdims=True)


def block_bwd_kept(dh_out, p, cache):
    """oracle.block.block_bwd from a cache whose block input, q, k, v, attention output, residual,
    MLP pre-activation (and adaLN branch outputs) were kept in the block format; LayerNorm
    statistics are the forward's; the attention is that of the kept q, k and v."""
    H, ada = cache["H"], cache["kind"] == "adaln"
    B, S, D = cache["h"].shape
    stats = {}
    for n, x in (("1", cache["h"]), ("2", cache["h1"])):
        mu = x.mean(axis=-1, keepdims=True)
        rstd = cache["c_ln" + n][1]
        xhat = (kept(x) - mu) * rstd
        u = xhat * (1.0 + cache["sc" + n]) + _shift(cache, n) if ada else xhat * p[f"ln{n}_w"] + p[f"ln{n}_b"]
        stats[n] = (xhat, rstd, u)
    qkv = kept(np.concatenate([blk.merge_heads(cache[n]) for n in "qkv"], axis=-1))
    q, k, v = (blk.split_heads(qkv[..., i * D:(i + 1) * D], H) for i in range(3))
    O, z = kept(cache["O"]), kept(cache["z"])
    flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    g = {n: np.zeros_like(t) for n, t in p.items()}
    dm, dgate2 = (dh_out * cache["g2"], (dh_out * kept(cache["m_out"])).sum(1)) if ada else (dh_out, None)
    g["w_fc2"], g["b_fc2"] = flat(dm).T @ flat(blk.gelu(z)), flat(dm).sum(0)
    dz = (dm @ p["w_fc2"]) * blk.gelu_grad(z)
    g["w_fc1"], g["b_fc1"] = flat(dz).T @ flat(stats["2"][2]), flat(dz).sum(0)
    du2 = dz @ p["w_fc1"]
    if ada:
        dscale2, dshift2 = (du2 * stats["2"][0]).sum(1), du2.sum(1)
        dx = blk.ln_bwd(du2 * (1.0 + cache["sc2"]), stats["2"][:2], None)[0]
    else:
        dx, g["ln2_w"], g["ln2_b"] = blk.ln_bwd(du2, stats["2"][:2], p["ln2_w"])
    dh1 = dh_out + dx
    da, dgate1 = (dh1 * cache["g1"], (dh1 * kept(cache["a_out"])).sum(1)) if ada else (dh1, None)
    g["w_o"], g["b_o"] = flat(da).T @ flat(O), flat(da).sum(0)
    d3 = _kept_attention_bwd(q, k, v, blk.split_heads(da @ p["w_o"], H))
    dqkv = np.concatenate([blk.merge_heads(t) for t in d3], axis=-1)
    g["w_qkv"], g["b_qkv"] = flat(dqkv).T @ flat(stats["1"][2]), flat(dqkv).sum(0)
    du = dqkv @ p["w_qkv"]
    dcond = None
    if ada:
        dmod = np.concatenate([du.sum(1), (du * stats["1"][0]).sum(1), dgate1, dshift2, dscale2, dgate2], axis=-1)
        dx = blk.ln_bwd(du * (1.0 + cache["sc1"]), stats["1"][:2], None)[0]
        g["w_ada"], g["b_ada"], dcond = dmod.T @ cache["cond"], dmod.sum(0), dmod @ p["w_ada"]
    else:
        dx, g["ln1_w"], g["ln1_b"] = blk.ln_bwd(du, stats["1"][:2], p["ln1_w"])
    return dh1 + dx, g, dcond


def stack_bwd_kept(dh, params64, caches):
    """oracle.stack.stack_bwd with block_bwd_kept."""
    grads, dcond = [None] * len(params64), None
    for i in reversed(range(len(params64))):
        dh, grads[i], dc = block_bwd_kept(dh, params64[i], caches[i])
        dcond = dc if dcond is None or dc is None else dcond + dc
    return dh, grads, dcond


def _linear8(x, w, b):
    """Rows of x (B, S, K) and of w quantised, their product, bias."""
    xq, xs = quant_rows(x.reshape(-1, x.shape[-1]))
    wq, ws = quant_rows(w)
    return linear(xq, xs, wq, ws, b).reshape(*x.shape[:-1], w.shape[0])


def block_fwd8(h, p, H, eps, kind="preln", cond=None):
    """oracle.block.block_fwd with its four linear layers on 8-bit rows."""
    D = h.shape[-1]
    ada = kind == "adaln"
    if ada:
        sh1, sc1, g1, sh2, sc2, g2 = blk._mod_chunks(p, cond)[0]
        u = blk.ln_fwd(h, None, None, eps)[0] * (1.0 + sc1) + sh1
    else:
        u = blk.ln_fwd(h, p["ln1_w"], p["ln1_b"], eps)[0]
    qkv = _linear8(u, p["w_qkv"], p["b_qkv"])
    O = blk.merge_heads(blk.attention_fwd(*(blk.split_heads(qkv[..., i * D:(i + 1) * D], H) for i in range(3))))
    a = _linear8(O, p["w_o"], p["b_o"])
    h1 = h + (g1 * a if ada else a)
    n2 = blk.ln_fwd(h1, None, None, eps)[0] * (1.0 + sc2) + sh2 if ada else blk.ln_fwd(h1, p["ln2_w"], p["ln2_b"], eps)[0]
    m = _linear8(blk.gelu(_linear8(n2, p["w_fc1"], p["b_fc1"])), p["w_fc2"], p["b_fc2"])
    return h1 + (g2 * m if ada else m)
