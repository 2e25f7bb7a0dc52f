"""Eight-bit activations in fp64: the two code formats, the linear layer on codes, and the weight
gradient from a checkpoint.  Plain formulas, no code shared with the GPU path.

Row format: q = 127 x / max|x| to the nearest integer (halves to even), value q * fl32(max|x| / 127).
Block format: 2^e per 32 channels, e the smallest integer in [-126, 121] with max|x| <= 127 2^e,
q = x 2^-e to the nearest integer within +-127, value q 2^e."""
from __future__ import annotations

import numpy as np
from scipy.special import erfc

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
