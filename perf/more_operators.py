"""Performance cases of the operators around and inside a block that is put together from single calls:

* ``rotary``   rotary positions of several axes on the heads of queries and keys (sr_rotary): every token turns by
               its own place on the token grid, the routed ones by the place that their index names;
* ``norm``     the residual step between two blocks (sr_residual_norm_fwd, sr_residual_norm_bwd): norm of the branch
               output, dropout, gate and residual scale, the sum, and the next branch's norm with its modulation;
* ``dropout``  dropout whose mask is drawn from a counter and never stored (sr_dropout), on values and gradients;
* ``f8``       the linear layer on 8-bit floating point with a power of two per block of 128 (sr_quantize_f8,
               sr_linear_f8): the tokens quantised and multiplied, or, for training, the input's and the
               weight's gradients.

B samples of S tokens; D channels; sizes are those of the forecaster's grids (16 x 32, 64 x 128, 90 x 180 tokens, widths 256 to
1024, MLP four times as wide), with odd ones among them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False   # False: the plain forms in elementary torch operations; True: the library's calls


def _rotary(B, S, heads, hd, grid, pairs, **kw):
    """grid and pairs as "90x180": tokens and channel pairs along each axis, slowest axis first."""
    c = dict(op="rotary", B=B, S=S, heads=heads, hd=hd, grid=grid, pairs=pairs, halves=True, routed=False,
             inverse=False, frame=0, dtype="bf16")
    c.update(kw)
    return c


def _norm(B, S, D, **kw):
    """post: norm of the branch output; mod: gate, shift and scale per sample; ls: a residual scale per channel;
    affine: weights of the norms; step: forward and backward."""
    c = dict(op="norm", B=B, S=S, D=D, rms=False, post=True, mod=False, ls=True, affine=True, p=0.0, step=False,
             dtype="bf16", stream="f32")
    c.update(kw)
    return c


def _dropout(M, N, **kw):
    c = dict(op="dropout", M=M, N=N, p=0.1, resid=False, group=0, dtype="bf16")
    c.update(kw)
    return c


def _f8(M, N, K, **kw):
    c = dict(op="f8", M=M, N=N, K=K, step=False, gelu=False, dtype="bf16")
    c.update(kw)
    return c


def listed():
    out = []

    def add(name, c):
        out.append(dict(c, name=name))

    # the queries of one token of a new frame: latency
    add("rotary_token", _rotary(1, 1, 16, 64, "4x16x32", "8x12x12", frame=3))
    # queries and keys of the routed tokens at 0.25 deg, a quarter of 90 x 180, side by side
    add("rotary_routed_025", _rotary(1, 4050, 32, 64, "90x180", "16x16", routed=True))
    # gradient of the keys of four frames of 64 x 128 tokens, two samples; neighbouring channels are the pairs
    add("rotary_frames", _rotary(2, 32768, 8, 128, "4x64x128", "16x24x24", halves=False, inverse=True))
    # one token of a forecast between two blocks: latency
    add("norm_token", _norm(1, 1, 1024))
    # training at 5.625 deg, eight samples, modulated blocks with dropout
    add("norm_step_5625", _norm(8, 512, 1024, mod=True, affine=False, p=0.1, step=True))
    # training at 0.25 deg, all tokens of a dense block, fp32 residual stream
    add("norm_step_025", _norm(1, 16200, 1024, rms=True, step=True))
    # an odd head of channels in the fp32 mode, added to what it updates
    add("dropout_odd_f32", _dropout(2013, 277, resid=True, dtype="f32"))
    # the MLP's hidden layer of a dense block at 0.25 deg
    add("dropout_025", _dropout(16200, 4096))
    # one token through the first MLP product: latency
    add("f8_token", _f8(1, 4096, 1024, gelu=True))
    # the forecaster's head: 69 variables on 2 x 2 points a token, width 256, ragged tokens, fp32 results
    add("f8_head", _f8(4083, 276, 256, dtype="f32"))
    # a dense block at 0.25 deg: the first MLP product with its GELU
    add("f8_025", _f8(16200, 4096, 1024, gelu=True))
    # training at 0.25 deg: both gradients of the second MLP product
    add("f8_step_025", _f8(16200, 1024, 4096, step=True))
    return out


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def size(lo, hi, unit):   # mostly whole units, odd ones among them
        return log_int(lo, hi) if rng.random() < 0.3 else unit * log_int(max(1, lo // unit), hi // unit)

    dtype = rng.choice(["bf16", "bf16", "f32"])
    op = rng.choice(["rotary", "norm", "norm", "dropout", "f8", "f8"])
    while True:
        if op == "rotary":
            hd = rng.choice([32, 64, 80, 96, 128, 2 * log_int(4, 64)])
            axes = rng.choice([1, 2, 3])
            cuts = sorted(rng.randint(1, hd // 2) for _ in range(axes))
            pairs = [b - a for a, b in zip([0] + cuts, cuts)]
            grid = [log_int(1, 200) for _ in range(axes)]
            L = math.prod(grid)
            routed = rng.random() < 0.5
            c = _rotary(log_int(1, 4), log_int(1, L) if routed else L, log_int(1, 32), hd, "x".join(map(str, grid)),
                        "x".join(map(str, pairs)), halves=rng.random() < 0.5, routed=routed,
                        inverse=rng.random() < 0.5, frame=rng.randint(0, 1000), dtype=dtype)
            if L <= 1 << 17 and c["B"] * c["S"] * c["heads"] * hd * (2 if dtype == "f32" else 1) <= 2 * 32768 * 1024:
                return c
        elif op == "norm":
            c = _norm(log_int(1, 8), log_int(1, 8192), size(32, 4096, 64), rms=rng.random() < 0.5,
                      post=rng.random() < 0.7, mod=rng.random() < 0.5, ls=rng.random() < 0.5,
                      affine=rng.random() < 0.5, p=rng.choice([0.0, 0.0, 0.1, 0.25]), step=rng.random() < 0.6,
                      dtype=dtype)
            c["stream"] = "f32" if c["step"] else rng.choice(["f32", dtype])   # training keeps the stream in fp32
            if c["B"] * c["S"] * c["D"] * (2 if dtype == "f32" else 1) <= 16200 * 1024:
                return c
        elif op == "dropout":
            c = _dropout(log_int(1, 16200), size(8, 4096, 8), p=rng.choice([0.0, 0.05, 0.1, 0.5]),
                         resid=rng.random() < 0.5, group=rng.choice([0, 0, 0, 1, log_int(1, 512)]), dtype=dtype)
            if c["M"] * c["N"] * (2 if dtype == "f32" else 1) * (2 if c["resid"] else 1) <= 16200 * 4096:
                return c
        else:
            c = _f8(log_int(1, 16200), size(16, 4096, 64), size(32, 4096, 64), step=rng.random() < 0.4, dtype=dtype)
            c["gelu"] = not c["step"] and rng.random() < 0.4
            if c["M"] * c["N"] * c["K"] <= 8192 * 1024 * 4096:
                return c


# ------------------------------------------------------------------------------ inputs

BLOCK = 128
SEED, STEP = 0x5EED, 11   # of the dropout's draws
EPS = 1e-6


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _ints(text):
    return [int(t) for t in text.split("x")]


def _up(n, m):
    return -(-n // m) * m


def _tokens(gen, M, N):
    """Activations: unit normals, some channels several times larger than the rest, tokens of unequal size."""
    x = torch.randn((M, N), generator=gen, device="cuda")
    ch = torch.exp(0.5 * torch.randn((1, N), generator=gen, device="cuda"))
    tok = torch.exp(0.3 * torch.randn((M, 1), generator=gen, device="cuda"))
    return x.mul_(ch).mul_(tok)


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    c, gen = case, _gen(seed)
    s, dt = dict(c), _dtype(c["dtype"])

    def vec(n, scale=0.1, mean=0.0):
        return mean + scale * torch.randn(n, generator=gen, device="cuda")

    if c["op"] == "rotary":
        M, L = c["B"] * c["S"], math.prod(_ints(c["grid"]))
        s["x"] = _tokens(gen, M, c["heads"] * c["hd"]).to(dt)
        if c["routed"]:   # one ascending draw of S of the L tokens per sample
            key = torch.rand((c["B"], L), generator=gen, device="cuda")
            s["idx"] = key.argsort(1)[:, : c["S"]].sort(1).values.to(torch.int32).contiguous()
        s["y"] = _empty(s["x"].shape, dt)
        if own:
            from paper_2607_02829_amd import abi
            axes = len(_ints(c["grid"]))
            s["rot"] = abi.SrRotary(grid=_ints(c["grid"]), pairs=_ints(c["pairs"]),
                                    layout=abi.SR_ROT_HALVES if c["halves"] else abi.SR_ROT_NEIGHBOURS, base=10000.0,
                                    origin=[float(c["frame"])] + [0.0] * (axes - 1))
        return s
    if c["op"] == "norm":
        B, M, D, st = c["B"], c["B"] * c["S"], c["D"], _dtype(c["stream"])
        s["x"], s["y"] = (2.0 * _tokens(gen, M, D)).to(st), _tokens(gen, M, D).to(dt)
        w = {}
        if c["affine"]:
            w["pre_w"], w["pre_b"] = vec(D, 0.1, 1.0).to(dt), vec(D).to(dt)
            if c["post"]:
                w["post_w"], w["post_b"] = vec(D, 0.1, 1.0).to(dt), vec(D).to(dt)
            if c["rms"]:
                w = {k: v for k, v in w.items() if k.endswith("_w")}
        if c["ls"]:
            w["res_scale"] = vec(D, 0.05, 0.2).to(dt)
        if c["mod"]:   # as the conditioning's product leaves them: one row of 6 D per sample, half of it this branch's
            s["mods"] = vec((B, 6 * D), 0.3)
            w["gate"], w["shift"], w["scale"] = s["mods"][:, :D], s["mods"][:, D:2 * D], s["mods"][:, 2 * D:3 * D]
        s["w"] = w
        s["x1"], s["u"] = _empty((M, D), st), _empty((M, D), dt)
        if c["step"]:
            s["dx1"], s["du"] = (0.05 * _tokens(gen, M, D)).to(st), (0.05 * _tokens(gen, M, D)).to(dt)
            s["stats"], s["dx"], s["dy"] = _empty((4, M), torch.float32), _empty((M, D), st), _empty((M, D), dt)
            s["g"] = {k: _empty((B, D) if v.dim() == 2 else (D,), torch.float32) for k, v in w.items()}
        if own:
            from paper_2607_02829_amd import abi
            s["cfg"] = abi.SrResidualNorm(
                B=B, S=c["S"], D=D, dtype=abi.SR_BF16 if c["dtype"] == "bf16" else abi.SR_F32,
                stream_dtype=abi.SR_BF16 if c["stream"] == "bf16" else abi.SR_F32,
                norm=abi.SR_NORM_RMS if c["rms"] else abi.SR_NORM_LAYER, post=int(c["post"]), eps=EPS, mod_stride=6 * D,
                drop=abi.SrDrop(p=c["p"], seed=SEED, step=STEP))
            s["params"] = abi.residual_norm_params(**w)
            if c["step"]:
                s["grads"] = abi.residual_norm_grads(**s["g"])
                s["scratch"] = _empty((max(abi.sr_residual_norm_scratch_bytes(s["cfg"]), 16),), torch.uint8)
        return s
    if c["op"] == "dropout":
        s["x"], s["y"] = _tokens(gen, c["M"], c["N"]).to(dt), _empty((c["M"], c["N"]), dt)
        s["r"] = _tokens(gen, c["M"], c["N"]).to(dt) if c["resid"] else None
        if own:
            from paper_2607_02829_amd import abi
            s["drop"] = abi.SrDrop(p=c["p"], seed=SEED, step=STEP, group=c["group"])
        return s
    M, N, K = c["M"], c["N"], c["K"]
    s["w"] = (torch.randn((N, K), generator=gen, device="cuda") / math.sqrt(K)).to(dt)
    s["x"] = _tokens(gen, M, K).to(dt)
    if c["step"]:
        s["dy"] = (0.05 * _tokens(gen, M, N)).to(dt)
    else:
        s["bias"] = vec(N).to(dt)
    if own:   # the weight's codes, and with a step those that the forward kept of its input
        from paper_2607_02829_amd import abi
        e = abi.SR_BF16 if c["dtype"] == "bf16" else abi.SR_F32
        s["wq"] = abi.f8_buffers(N, K, transposed=c["step"], rows=not c["step"])
        abi.sr_quantize_f8(abi.SR_F8_TILE, e, N, K, s["w"], K, *s["wq"])
        s["xq"] = abi.f8_buffers(M, K, transposed=c["step"], rows=not c["step"])
        if c["step"]:
            abi.sr_quantize_f8(abi.SR_F8_ROW, e, M, K, s["x"], K, *s["xq"])
            s["dyq"] = abi.f8_buffers(M, N, transposed=True, rows=True)
            s["dx"], s["dw"] = _empty((M, K), dt), _empty((N, K), torch.float32)
            n = max(abi.sr_linear_f8_scratch_bytes(M, K, N), abi.sr_linear_f8_scratch_bytes(N, K, M))
        else:
            s["y"] = _empty((M, N), dt)
            n = abi.sr_linear_f8_scratch_bytes(M, N, K)
        s["scratch"] = _empty((max(n, 16),), torch.uint8)
    else:
        s["wv"] = _f8_values(s["w"].float(), BLOCK, BLOCK)
        if c["step"]:
            s["xv"] = _f8_values(s["x"].float(), BLOCK, 1)
    return s


# ------------------------------------------------------------------------------ plain forms

_G = 0x9E3779B97F4A7C15


def _i64(v):
    """An unsigned 64-bit number as the signed one of the same bits."""
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >= 1 << 63 else v


def _shift(z, n):
    return (z >> n) & ((1 << (64 - n)) - 1)


def _mix(z):
    z = (z ^ _shift(z, 30)) * _i64(0xBF58476D1CE4E5B9)
    z = (z ^ _shift(z, 27)) * _i64(0x94D049BB133111EB)
    return z ^ _shift(z, 31)


def _plain_keep(p, M, N, group):
    """(keep [M, N] or [M, 1], the factor of what is kept)."""
    t = int(round(p * 65536))
    key = _mix(torch.tensor([_i64(SEED + (STEP + 1) * _G)], device="cuda"))
    e = torch.arange(M, device="cuda").view(M, 1)
    e = e // group if group else e * N + torch.arange(N, device="cuda")
    word = _mix(key + ((e >> 2) + 1) * _i64(_G))
    return ((word >> (16 * (e & 3))) & 0xFFFF) >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0


def _plain_norm(x, rms):
    if not rms:
        x = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * rstd, rstd


def _plain_norm_grad(g, xhat, rstd, rms):
    d = g - xhat * (g * xhat).mean(1, keepdim=True)
    if not rms:
        d = d - g.mean(1, keepdim=True)
    return d * rstd


def _run_plain_norm(s):
    B, S, D, rms, dt, st = s["B"], s["S"], s["D"], s["rms"], _dtype(s["dtype"]), _dtype(s["stream"])
    w = {k: v.float() for k, v in s["w"].items()}
    rows = {k: w[k].repeat_interleave(S, dim=0) for k in ("gate", "shift", "scale") if k in w}
    y = s["y"].float()
    n = y
    if s["post"]:
        yhat, yr = _plain_norm(y, rms)
        n = yhat * w.get("post_w", 1.0) + w.get("post_b", 0.0)
    f = None
    if s["p"] > 0:
        keep, f = _plain_keep(s["p"], B * S, D, 0)
        n = torch.where(keep, n * f, 0.0)
    a = w.get("res_scale", 1.0)
    x1 = (s["x"].float() + rows.get("gate", 1.0) * a * n).to(st)
    v, vr = _plain_norm(x1.float(), rms)
    t = v * w.get("pre_w", 1.0) + w.get("pre_b", 0.0)
    u = t * (1.0 + rows.get("scale", 0.0)) + rows.get("shift", 0.0)
    out = {"x1": x1, "u": u.to(dt)}
    if not s["step"]:
        return out
    du = s["du"].float()

    def samples(z):
        return z.view(B, S, D).sum(1)

    g = {}
    if "scale" in w:
        g["shift"], g["scale"] = samples(du), samples(du * t)
    dt_ = du * (1.0 + rows.get("scale", 0.0))
    if "pre_w" in w:
        g["pre_w"] = (dt_ * v).sum(0)
    if "pre_b" in w:
        g["pre_b"] = dt_.sum(0)
    dx = s["dx1"].float() + _plain_norm_grad(dt_ * w.get("pre_w", 1.0), v, vr, rms)
    if "gate" in w:
        g["gate"] = samples(dx * a * n)
    if "res_scale" in w:
        g["res_scale"] = (dx * rows.get("gate", 1.0) * n).sum(0)
    dn = dx * rows.get("gate", 1.0) * a
    if f is not None:
        dn = torch.where(keep, dn * f, 0.0)
    if "post_w" in w:
        g["post_w"] = (dn * yhat).sum(0)
    if "post_b" in w:
        g["post_b"] = dn.sum(0)
    dy = _plain_norm_grad(dn * w.get("post_w", 1.0), yhat, yr, rms) if s["post"] else dn
    return dict(out, dx=dx.to(st), dy=dy.to(dt), **{"d_" + k: v for k, v in g.items()})


def _run_plain_rotary(s):
    B, S, H, hd = s["B"], s["S"], s["heads"], s["hd"]
    grid, pairs = _ints(s["grid"]), _ints(s["pairs"])
    at = s["idx"].long() if s["routed"] else torch.arange(S, device="cuda").expand(B, S)
    angles = []
    for a in reversed(range(len(grid))):
        place = (at % grid[a]).double() + (float(s["frame"]) if a == 0 else 0.0)
        at = at // grid[a]
        j = torch.arange(pairs[a], device="cuda", dtype=torch.float64)
        angles.insert(0, place.unsqueeze(2) * torch.pow(10000.0, -j / max(pairs[a], 1)))
    t = torch.cat(angles, 2).view(B * S, 1, -1)
    co, si = torch.cos(t).float(), torch.sin(t).float()
    if s["inverse"]:
        si = -si
    x, P = s["x"].float().view(B * S, H, hd), t.shape[2]
    if s["halves"]:
        lo, hi = x[..., :P], x[..., P:2 * P]
        y = torch.cat([lo * co - hi * si, hi * co + lo * si, x[..., 2 * P:]], 2)
    else:
        lo, hi = x[..., 0:2 * P:2], x[..., 1:2 * P:2]
        y = torch.stack([lo * co - hi * si, hi * co + lo * si], 3).view(B * S, H, 2 * P)
        y = torch.cat([y, x[..., 2 * P:]], 2)
    return {"y": y.view(B * S, H * hd).to(_dtype(s["dtype"]))}


def _f8_values(x, rows, cols):
    """What the codes of x stand for: e4m3 with a power of two per block of rows x cols, the smallest that keeps the
    block within 448."""
    M, N = x.shape
    t = x.new_zeros((_up(M, rows), _up(N, cols)))
    t[:M, :N] = x
    t = t.view(t.shape[0] // rows, rows, t.shape[1] // cols, cols)
    m, e = torch.frexp(t.abs().amax((1, 3), keepdim=True))
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(-126, 119)
    q = torch.ldexp(t, -e).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()
    return torch.ldexp(q, e).reshape(t.shape[0] * rows, -1)[:M, :N]


def _run_plain(s):
    if s["op"] == "rotary":
        return _run_plain_rotary(s)
    if s["op"] == "norm":
        return _run_plain_norm(s)
    dt = _dtype(s["dtype"])
    if s["op"] == "dropout":
        keep, f = _plain_keep(s["p"], s["M"], s["N"], s["group"])
        y = torch.where(keep, s["x"].float() * f, 0.0)
        return {"y": (y + s["r"].float() if s["resid"] else y).to(dt)}
    if s["step"]:
        dy = s["dy"].float()
        dx = torch.matmul(_f8_values(dy, 1, BLOCK), s["wv"])
        return {"dx": dx.to(dt), "dw": torch.matmul(_f8_values(dy, BLOCK, 1).t(), s["xv"])}
    y = torch.matmul(_f8_values(s["x"].float(), 1, BLOCK), s["wv"].t()) + s["bias"].float()
    if s["gelu"]:
        y = 0.5 * y * torch.erfc(y * -math.sqrt(0.5))
    return {"y": y.to(dt)}


# ------------------------------------------------------------------------------ the library's calls


def _run_own(s):
    from paper_2607_02829_amd import abi
    dt = abi.SR_BF16 if s["dtype"] == "bf16" else abi.SR_F32
    if s["op"] == "rotary":
        n = s["heads"] * s["hd"]
        abi.sr_rotary(s["rot"], int(s["inverse"]), dt, s["B"], s["S"], s["heads"], s["hd"], s["x"], n, s.get("idx"), 0,
                      s["y"], n)
        return {"y": s["y"]}
    if s["op"] == "norm":
        abi.sr_residual_norm_fwd(s["cfg"], s["params"], s["x"], s["y"], s["x1"], s["u"], None, None, s.get("stats"))
        out = {"x1": s["x1"], "u": s["u"]}
        if s["step"]:
            abi.sr_residual_norm_bwd(s["cfg"], s["params"], s["x1"], s["y"], s["stats"], s["dx1"], s["du"], s["dx"],
                                     s["dy"], s["grads"], s["scratch"])
            out.update(dx=s["dx"], dy=s["dy"], **{"d_" + k: v for k, v in s["g"].items()})
        return out
    if s["op"] == "dropout":
        abi.sr_dropout(s["drop"], dt, s["M"], s["N"], s["x"], s["r"], s["y"])
        return {"y": s["y"]}
    M, N, K, none = s["M"], s["N"], s["K"], abi.SR_ACT_NONE
    if s["step"]:
        dq, de, dqt, det = s["dyq"]
        abi.sr_quantize_f8(abi.SR_F8_ROW, dt, M, N, s["dy"], N, dq, de, dqt, det)
        abi.sr_linear_f8(dt, none, M, K, N, dq, de, s["wq"][2], s["wq"][3], None, s["dx"], s["scratch"])
        abi.sr_linear_f8(abi.SR_F32, none, N, K, M, dqt, det, s["xq"][2], s["xq"][3], None, s["dw"], s["scratch"])
        return {"dx": s["dx"], "dw": s["dw"]}
    xq, xe = s["xq"][:2]
    abi.sr_quantize_f8(abi.SR_F8_ROW, dt, M, K, s["x"], K, xq, xe, None, None)
    abi.sr_linear_f8(dt, abi.SR_ACT_GELU if s["gelu"] else none, M, N, K, xq, xe, s["wq"][0], s["wq"][1], s["bias"],
                     s["y"], s["scratch"])
    return {"y": s["y"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    if c["op"] == "rotary":
        M = c["B"] * c["S"]
        n = M * c["heads"] * c["hd"]
        return {"bytes": 2 * e * n + (4 * M if c["routed"] else 0), "flops": 3 * n}
    if c["op"] == "norm":
        n, st = c["B"] * c["S"] * c["D"], 2 if c["stream"] == "bf16" else 4
        # x and y, x1 and u; with a step dx1 and du, dx and dy too
        return {"bytes": (4 if c["step"] else 2) * n * (st + e), "flops": (40 if c["step"] else 15) * n}
    if c["op"] == "dropout":
        return {"bytes": c["M"] * c["N"] * e * (3 if c["resid"] else 2), "flops": 2 * c["M"] * c["N"]}
    M, N, K = c["M"], c["N"], c["K"]
    if c["step"]:   # dy and the codes of x and w; dx and dw
        return {"bytes": e * M * N + M * K + N * K + e * M * K + 4 * N * K, "flops": 4 * M * N * K}
    return {"bytes": e * M * K + N * K + e * N + e * M * N, "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------ 64-bit results


def _draws(p, M, N, group):
    """keep as an array of unsigned arithmetic, and the factor."""
    def mix(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    gamma = np.uint64(_G)
    with np.errstate(over="ignore"):
        key = mix(np.array([SEED], np.uint64) + np.uint64(STEP + 1) * gamma)
        count = (M + group - 1) // group if group else M * N
        words = mix(key + np.arange(1, (count + 3) // 4 + 1, dtype=np.uint64) * gamma)
    kept = words.view(np.uint16)[:count].astype(np.int32) >= int(round(p * 65536))   # little-endian: the lowest bits first
    kept = np.repeat(kept, group)[:M, None] if group else kept.reshape(M, N)
    t = int(round(p * 65536))
    return torch.from_numpy(kept).cuda(), 65536.0 / (65536 - t) if t < 65536 else 0.0


def _e4m3(x, rows, cols):
    """The nearest values of e4m3 times each block's power of two."""
    M, N = x.shape
    out = torch.zeros((_up(M, rows), _up(N, cols)), dtype=torch.float64, device=x.device)
    out[:M, :N] = x
    b = out.unfold(0, rows, rows).unfold(1, cols, cols)
    top = b.abs().amax((2, 3))[:, :, None, None]
    e = torch.ceil(torch.log2((top / 448.0).clamp_min(2.0 ** -126)))
    e = e + (top > 448.0 * torch.exp2(e)).double()                   # a border that the logarithm rounded over
    e = e - ((top <= 448.0 * torch.exp2(e - 1.0)) & (e > -126.0)).double()
    e = e.clamp(max=119.0)
    scale = torch.exp2(e)
    v = b / scale
    size = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))    # of an fp32 value over a power of two: far from rounding up
    unit = torch.exp2(size - 3.0)
    v = (torch.round(v / unit) * unit).clamp(-448.0, 448.0) * scale
    return v.permute(0, 2, 1, 3).reshape(out.shape)[:M, :N].contiguous()


def _exact_norm(c, s):
    B, S, D = c["B"], c["S"], c["D"]
    one, zero = torch.ones((), dtype=torch.float64, device="cuda"), torch.zeros((), dtype=torch.float64, device="cuda")
    leaf = {k: v.double().reshape((B, 1, D) if v.dim() == 2 else (D,)).contiguous().requires_grad_(c["step"])
            for k, v in s["w"].items()}
    x = s["x"].double().view(B, S, D).requires_grad_(c["step"])
    y = s["y"].double().view(B, S, D).requires_grad_(c["step"])

    def norm(z, w, b):
        if not c["rms"]:
            z = z - z.sum(-1, keepdim=True) / D
        return z / torch.sqrt(z.square().sum(-1, keepdim=True) / D + EPS) * leaf.get(w, one) + leaf.get(b, zero)

    n = norm(y, "post_w", "post_b") if c["post"] else y
    if c["p"] > 0:
        keep, f = _draws(c["p"], B * S, D, 0)
        n = n * (keep.view(B, S, D).double() * f)
    x1 = x + leaf.get("gate", one) * leaf.get("res_scale", one) * n
    kept = x1 + (x1.detach().to(_dtype(c["stream"])).double() - x1.detach()) if c["stream"] == "bf16" else x1   # as it is stored
    u = norm(kept, "pre_w", "pre_b") * (1.0 + leaf.get("scale", zero)) + leaf.get("shift", zero)
    out = {"x1": x1.detach().view(-1, D), "u": u.detach().view(-1, D)}
    if c["step"]:
        ins = [x, y] + list(leaf.values())
        g = torch.autograd.grad([x1, u], ins, [s["dx1"].double().view(B, S, D), s["du"].double().view(B, S, D)])
        out.update(dx=g[0].view(-1, D), dy=g[1].view(-1, D))
        out.update({"d_" + k: v.reshape(s["g"][k].shape) for k, v in zip(leaf, g[2:])})
    return out


def _exact_rotary(c, s):
    """As a product of complex numbers."""
    grid, pairs = _ints(c["grid"]), _ints(c["pairs"])
    B, S, H, hd, P = c["B"], c["S"], c["heads"], c["hd"], sum(_ints(c["pairs"]))
    at = s["idx"].cpu().numpy() if c["routed"] else np.broadcast_to(np.arange(S), (B, S))
    places = np.unravel_index(at.reshape(-1).astype(np.int64), grid)
    turn = np.concatenate([(places[a][:, None] + (c["frame"] if a == 0 else 0))
                           * np.float64(10000.0) ** (-np.arange(pairs[a]) / max(pairs[a], 1)) for a in range(len(grid))], 1)
    z = torch.polar(torch.ones(turn.shape, dtype=torch.float64), torch.from_numpy(-turn if c["inverse"] else turn)).cuda()
    x = s["x"].double().view(B * S, H, hd)
    a, b = (slice(0, P), slice(P, 2 * P)) if c["halves"] else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    r = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * z[:, None, :]
    y = x.clone()
    y[..., a], y[..., b] = r.real, r.imag
    return {"y": y.view(B * S, H * hd)}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rotary":
        return _exact_rotary(c, s)
    if c["op"] == "norm":
        return _exact_norm(c, s)
    if c["op"] == "dropout":
        keep, f = _draws(c["p"], c["M"], c["N"], c["group"])
        y = s["x"].double() * keep.double() * f
        return {"y": y + s["r"].double() if c["resid"] else y}
    w = _e4m3(s["w"].double(), BLOCK, BLOCK)
    if c["step"]:
        dy, x = s["dy"].double(), s["x"].double()
        return {"dx": _e4m3(dy, 1, BLOCK) @ w, "dw": _e4m3(dy, BLOCK, 1).t().contiguous() @ _e4m3(x, BLOCK, 1)}
    y = _e4m3(s["x"].double(), 1, BLOCK) @ w.t().contiguous() + s["bias"].double()
    return {"y": y * torch.special.ndtr(y) if c["gelu"] else y}
