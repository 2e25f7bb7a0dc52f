"""Plain 64-bit forms of the operators around and inside a block: rotary positions, dropout from a counter, the residual
step with its norms (forward and backward), and 8-bit floating point with a power of two per block of 128."""
from __future__ import annotations

import numpy as np

from .select import GAMMA, mix64

# ---------------------------------------------------------------- rotary positions


def rotary(x, idx, grid, pairs, neighbours=False, base=10000.0, origin=None, step=None, freqs=None, inverse=False):
    """x [B,S,heads,hd] float64, idx [B,S] or [1,S] or None -> the turned heads, and the largest angle."""
    B, S, H, hd = x.shape
    n = len(grid)
    origin, step = origin or [0.0] * n, step or [1.0] * n
    at = np.broadcast_to(np.arange(S) if idx is None else idx, (B, S)).astype(np.int64)
    places = np.unravel_index(at, grid)
    p0, turns = 0, []
    for a in range(n):
        f = np.asarray(freqs[p0:p0 + pairs[a]]) if freqs is not None else float(base) ** (-np.arange(pairs[a]) / max(pairs[a], 1))
        turns.append((origin[a] + step[a] * places[a])[..., None] * f)
        p0 += pairs[a]
    t = np.concatenate(turns, -1)[:, :, None, :]
    c, s = np.cos(t), np.sin(-t if inverse else t)
    P = p0
    lo, hi = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if neighbours else (slice(0, P), slice(P, 2 * P))
    y = x.copy()
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., hi] * c + x[..., lo] * s
    return y, float(np.abs(t).max()) if P else 0.0


# ---------------------------------------------------------------- dropout


def drop_threshold(p) -> int:
    return int(np.rint(float(np.float32(p)) * 65536.0))


def drop_factor(p) -> float:
    t = drop_threshold(p)
    return float(np.float32(65536.0 / (65536 - t))) if t < 65536 else 0.0


def drop_keep(M, N, p, seed, step, first_row=0, group=0):
    """bool [M,N]: the values that stay."""
    with np.errstate(over="ignore"):
        key = mix64(np.array([seed], np.uint64) + np.array([step + 1 & (2 ** 64 - 1)], np.uint64) * GAMMA)
        row = np.uint64(first_row) + np.arange(M, dtype=np.uint64)
        if group:
            e = np.repeat((row // np.uint64(group))[:, None], N, 1)
        else:
            e = row[:, None] * np.uint64(N) + np.arange(N, dtype=np.uint64)
        word = mix64(key + (e // np.uint64(4) + np.uint64(1)) * GAMMA)
    return (word >> (np.uint64(16) * (e % np.uint64(4))) & np.uint64(0xFFFF)).astype(np.int64) >= drop_threshold(p)


# ---------------------------------------------------------------- residual step


def norm(z, rms, eps):
    mean = np.zeros(z.shape[:-1] + (1,)) if rms else z.mean(-1, keepdims=True)
    d = z - mean
    rstd = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return d * rstd, mean, rstd


def _norm_grad(g, zhat, rstd, rms):
    d = g - zhat * (g * zhat).mean(-1, keepdims=True)
    return rstd * (d if rms else d - g.mean(-1, keepdims=True))


def residual_norm(x, y, w, rms, post, eps, keep=None, factor=1.0, stored=None):
    """x, y [B,S,D] (y or None), w: parameters by name (gate, shift, scale [B,D]).  stored: x1 in the stream's type ->
    the x1 that the next norm reads.  Returns x1, u and what the backward needs."""
    def vec(k, fill):
        v = w.get(k)
        return fill if v is None else v[:, None, :] if v.ndim == 2 else v

    k = dict(x=x, y=y, w=w, rms=rms, post=post, keep=keep, factor=factor)
    if y is None:
        x1 = x
    else:
        n = y
        if post:
            k["yhat"], _, k["yrstd"] = norm(y, rms, eps)
            n = k["yhat"] * vec("post_w", 1.0) + vec("post_b", 0.0)
        if keep is not None:
            n = np.where(keep, n * factor, 0.0)
        k["n"] = n
        x1 = x + vec("gate", 1.0) * vec("res_scale", 1.0) * n
    kept = x1 if stored is None else stored(x1)
    k["xhat"], _, k["xrstd"] = norm(kept, rms, eps)
    k["t"] = k["xhat"] * vec("pre_w", 1.0) + vec("pre_b", 0.0)
    return x1, k["t"] * (1.0 + vec("scale", 0.0)) + vec("shift", 0.0), k


def residual_norm_bwd(k, dx1, du):
    """dx, dy, gradients by name, and the sums of the magnitudes that each of those adds up."""
    w, rms = k["w"], k["rms"]

    def vec(n, fill):
        v = w.get(n)
        return fill if v is None else v[:, None, :] if v.ndim == 2 else v

    g, mag = {}, {}

    def put(name, t, samples):
        axes = (1,) if samples else (0, 1)
        g[name], mag[name] = t.sum(axes), np.abs(t).sum(axes)

    dx = 0.0 if dx1 is None else dx1
    if du is not None:
        put("shift", du, True)
        put("scale", du * k["t"], True)
        d = du * (1.0 + vec("scale", 0.0))
        put("pre_w", d * k["xhat"], False)
        put("pre_b", d, False)
        dx = dx + _norm_grad(d * vec("pre_w", 1.0), k["xhat"], k["xrstd"], rms)
    dy = None
    if k["y"] is not None:
        a = vec("res_scale", 1.0)
        put("gate", dx * a * k["n"], True)
        put("res_scale", dx * vec("gate", 1.0) * k["n"], False)
        dn = dx * vec("gate", 1.0) * a
        if k["keep"] is not None:
            dn = np.where(k["keep"], dn * k["factor"], 0.0)
        dy = dn
        if k["post"]:
            put("post_w", dn * k["yhat"], False)
            put("post_b", dn, False)
            dy = _norm_grad(dn * vec("post_w", 1.0), k["yhat"], k["yrstd"], rms)
    return dx, dy, g, mag


# ---------------------------------------------------------------- 8-bit floating point

_VALUES = None


def e4m3_values():
    """float64 of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    global _VALUES
    if _VALUES is None:
        c = np.arange(256)
        e, m = (c >> 3) & 15, c & 7
        v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
        v = np.where(c >= 128, -v, v)
        v[0x7F] = v[0xFF] = np.nan
        _VALUES = v
    return _VALUES


def e4m3_codes(v):
    """Nearest code of each value, |v| <= 448, halves to the even code."""
    table = e4m3_values()[:127]                                   # 0 .. 448, ascending with the code
    a = np.abs(v)
    hi = np.searchsorted(table, a).clip(1, 126)
    lo = hi - 1
    dl, dh = a - table[lo], table[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    code = np.where(a == 0, 0, code)
    return (code + 128 * np.signbit(v)).astype(np.uint8)


def f8_quantize(x, tile=False):
    """x [R,C] float64 -> (codes [R,Cp] uint8, exponents [Cp/128,R] uint8 of e + 127, values [R,C])."""
    R, C = x.shape
    Cp, Rt = -(-C // 128) * 128, -(-R // 128) * 128
    z = np.zeros((Rt, Cp))
    z[:R, :C] = x
    b = z.reshape(Rt // 128, 128, Cp // 128, 128)
    with np.errstate(invalid="ignore"):
        top = np.abs(b).max((1, 3) if tile else 3, keepdims=True)
    top = np.broadcast_to(top, (Rt // 128, 128, Cp // 128, 1))
    bad = ~np.isfinite(top)
    m, e = np.frexp(np.where(bad, 1.0, top))
    e = np.clip(np.where(top == 0, -126, np.where(m > 0.875, e - 8, e - 9)), -126, 119)
    e = np.where(bad, 0, e)
    with np.errstate(invalid="ignore"):
        q = np.where(bad, 0x7F, e4m3_codes(np.clip(np.nan_to_num(b * 2.0 ** -e.astype(float)), -448, 448))).astype(np.uint8)
    vals = e4m3_values()[q] * 2.0 ** e.astype(float)
    q.reshape(Rt // 128, 128, Cp)[:, :, C:] = 0      # past a row's end, also in a block of NaN codes
    back = lambda t: t.reshape(Rt, -1)[:R]  # noqa: E731
    return back(q), (back(e) + 127).astype(np.uint8).T, back(vals)[:, :C]
