"""The column sums of sr_residual_norm_bwd row by row: whole numbers, whose sums are exact in every order, so that one row too few, too
many or twice shows; and numbers of the usual kind against a bound of each channel's own summands.

That bound, u = 2^-24.  A normed value is off by at most 194 u (1 + its magnitude) (32 u (1 + |mean| rstd) + 34 u of it, |mean| rstd
< 4), rounded up to 256 u; dx by 256 u of |dx1| and of rstd max|g| (1 + max|Norm|) over the row.  A channel's sum is formed from at most
128 + B summands one after another (a team's rows, 16 teams, the parts of a sample eight at most to each of 32 groups, the samples), so its own
roundings are at most (128 + B) u of its summands' magnitudes, and typically far less: in root mean square under 32 u."""
import numpy as np
import pytest

from oracle import block_ops as ob
from paper_2607_02829_amd import abi
from test_gpu_residual_norm import EPS, _setup

pytestmark = pytest.mark.gpu

U, C = 2.0 ** -24, 256.0

WHOLE = [
    # B, S, D, post, dtype, stream
    (1, 1, 1, True, "f32", "f32"), (1, 9000, 64, True, "bf16", "f32"), (2, 300, 1024, True, "bf16", "f32"), (1200, 2, 32, True, "bf16", "f32"),
    (1, 16200, 1024, True, "bf16", "f32"), (1, 16200, 96, False, "bf16", "bf16"), (8, 512, 1024, True, "bf16", "f32"),
    (1, 256, 1024, True, "bf16", "f32"), (1, 257, 1024, True, "bf16", "f32"), (1, 2049, 1024, True, "f32", "f32"), (3, 85, 600, True, "f32", "f32"),
    (33, 7, 300, True, "bf16", "bf16"), (31, 301, 130, True, "bf16", "f32"), (64, 129, 260, False, "bf16", "f32"), (1, 5003, 1023, True, "bf16", "f32"),
    (5, 77, 5, True, "f32", "f32"), (2, 333, 2, True, "bf16", "f32"), (1, 4099, 3, True, "f32", "f32"), (1, 2050, 2048, True, "bf16", "f32"),
    (1, 700, 4000, True, "bf16", "f32"), (2, 40, 8191, True, "f32", "f32"), (40, 65, 129, True, "bf16", "f32"), (1, 3001, 1500, True, "bf16", "bf16"),
    (300, 1, 512, True, "bf16", "f32"), (513, 9, 64, True, "f32", "f32"),
]


@pytest.mark.parametrize("c", WHOLE, ids=lambda c: "-".join(map(str, c)))
def test_whole_numbers(c):
    import torch
    B, S, D, post, dtype, stream = c
    M, dt, st = B * S, torch.bfloat16 if dtype == "bf16" else torch.float32, torch.bfloat16 if stream == "bf16" else torch.float32
    g = torch.Generator().manual_seed(B + S + D)
    ints = lambda n, *s: torch.randint(-n, n + 1, s, generator=g).float()  # noqa: E731
    x1, y, dx1, du = ints(3, M, D), ints(3, M, D), ints(3, M, D), ints(3, M, D)
    w = {"post_w": ints(2, D), "post_b": ints(2, D), "res_scale": ints(2, D), "pre_w": ints(2, D), "pre_b": ints(2, D)}
    mods = {n: ints(2, B, D + 3) for n in ("gate", "shift", "scale")}
    stats = torch.stack([ints(1, M), 2.0 ** ints(1, M), ints(1, M), 2.0 ** ints(1, M)])   # means, and reciprocal deviations of 1/2, 1 and 2
    cfg = abi.SrResidualNorm(B=B, S=S, D=D, dtype=abi.SR_BF16 if dtype == "bf16" else abi.SR_F32,
                             stream_dtype=abi.SR_BF16 if stream == "bf16" else abi.SR_F32, norm=abi.SR_NORM_LAYER, post=int(post), eps=EPS,
                             mod_stride=D + 3, drop=abi.SrDrop(p=0.5, seed=4, step=1))
    params = abi.residual_norm_params(**{n: v.to(dt).cuda() for n, v in w.items()}, **{n: v.cuda() for n, v in mods.items()})
    scratch = torch.full((abi.sr_residual_norm_scratch_bytes(cfg),), 0xFF, dtype=torch.uint8, device="cuda")
    grads = {n: torch.full((D,), float("nan"), device="cuda") for n in w}
    grads.update({n: torch.full((B, D), float("nan"), device="cuda") for n in mods})
    dx, dy = torch.empty((M, D), dtype=st, device="cuda"), torch.empty((M, D), dtype=dt, device="cuda")
    gs = abi.residual_norm_grads(**grads)
    xd, yd, dxd, dud, sd = x1.to(st).cuda(), y.to(dt).cuda(), dx1.to(st).cuda(), du.to(dt).cuda(), stats.cuda()
    w = {n: v.double().numpy() for n, v in w.items()}
    gate, scale = mods["gate"][:, :D].double().numpy(), 1.0 + mods["scale"][:, :D].double().numpy()
    stats = stats.double().numpy()
    samples = lambda t: t.reshape(B, S, D).sum(1)  # noqa: E731

    def same(name, want):
        assert np.abs(want).max() < 2.0 ** 22
        assert np.array_equal(grads[name].cpu().double().numpy(), want), (name, np.argwhere(grads[name].cpu().double().numpy() != want)[:5])

    # gradients of the norm before the next branch: du alone
    abi.sr_residual_norm_bwd(cfg, params, xd, None, sd, None, dud, dx, None, gs, scratch)
    d64 = du.double().numpy()
    v = (x1.double().numpy() - stats[2][:, None]) * stats[3][:, None]
    s1, s2 = samples(d64), samples(d64 * v)
    same("shift", s1)
    same("scale", w["pre_w"] * s2 + w["pre_b"] * s1)
    same("pre_w", (scale * s2).sum(0))
    same("pre_b", (scale * s1).sum(0))
    # gradients of the step: dx1 alone, which is dx; p = 1/2 doubles what it keeps
    scratch.fill_(0xFF)
    abi.sr_residual_norm_bwd(cfg, params, xd, yd, sd, dxd, None, dx, dy, gs, scratch)
    assert torch.equal(dx, dxd)
    d = dx1.double().numpy() * ob.drop_keep(M, D, 0.5, 4, 1) * 2.0
    n = (y.double().numpy() - stats[0][:, None]) * stats[1][:, None] if post else y.double().numpy()
    s3, s4 = samples(d), samples(d * n)
    t = w["post_w"] * s4 + w["post_b"] * s3 if post else s4
    same("gate", w["res_scale"] * t)
    same("res_scale", (gate * t).sum(0))
    same("post_w", (gate * w["res_scale"] * s4).sum(0) if post else np.zeros(D))
    same("post_b", (gate * w["res_scale"] * s3).sum(0) if post else np.zeros(D))


CASES = [
    # B, S, D, rms, post, names of the parameters, p, group, dtype, stream
    (1, 9000, 64, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.1, 0, "bf16", "f32"),
    (2, 300, 1024, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.1, 0, "bf16", "f32"),
    (1200, 2, 32, True, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.1, 2, "bf16", "f32"),
    (1, 4099, 1023, True, True, "post_w res_scale pre_w", 0.0, 0, "f32", "f32"),
    (3, 700, 2048, False, True, "post_w post_b pre_w pre_b gate", 0.2, 0, "bf16", "bf16"),
    (2, 1025, 300, False, False, "res_scale pre_w pre_b gate scale", 0.1, 0, "f32", "f32"),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", "_"))
def test_each_channel_by_its_own_summands(c):
    import torch
    B, S, D, rms, post, names, p, group, dtype, stream = c
    cfg, x, y, w, w64, keep, g = _setup(c)
    M, f = B * S, ob.drop_factor(p)
    params = abi.residual_norm_params(**w)
    xd, yd = x.cuda(), y.cuda()
    x1, u, stats = torch.empty_like(xd), torch.empty_like(yd), torch.empty((4, M), device="cuda")
    abi.sr_residual_norm_fwd(cfg, params, xd, yd, x1, u, stats=stats)
    dx1 = (0.3 * torch.randn((B, S, D), generator=g)).to(x.dtype)
    du = (0.3 * torch.randn((B, S, D), generator=g)).to(y.dtype)
    grads = {n: torch.full((B, D) if v.dim() == 2 else (D,), float("nan"), device="cuda") for n, v in w.items()}
    scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    abi.sr_residual_norm_bwd(cfg, params, x1, yd, stats, dx1.cuda(), du.cuda(), torch.empty_like(xd), torch.empty_like(yd),
                             abi.residual_norm_grads(**grads), scratch)
    _, _, k = ob.residual_norm(x.double().numpy(), y.double().numpy(), w64, rms, post, EPS, keep, f, stored=lambda _: x1.cpu().double().numpy())
    dx164, du64 = dx1.double().numpy(), du.double().numpy()
    _, _, want, mag = ob.residual_norm_bwd(k, dx164, du64)

    vec = lambda n, fill: np.broadcast_to(np.asarray(w64.get(n, fill), np.float64), (B, D) if n in ("gate", "shift", "scale") else (D,))  # noqa: E731
    per = lambda n, fill: vec(n, fill)[:, None, :] if n in ("gate", "shift", "scale") else vec(n, fill)  # noqa: E731
    top = lambda t: np.abs(t).max(-1, keepdims=True)  # noqa: E731
    e_v = C * U * (1.0 + np.abs(k["xhat"]))
    gin = du64 * (1.0 + per("scale", 0.0)) * per("pre_w", 1.0)
    dx, _, _, _ = ob.residual_norm_bwd(k, dx164, du64)
    e_dx = C * U * (np.abs(dx164) + k["xrstd"] * top(gin) * (1.0 + top(k["xhat"])))
    kp = 1.0 if keep is None else keep
    d, e_d = kp * f * np.abs(dx), kp * f * e_dx
    n = np.abs(k["yhat"] if post else y.double().numpy())
    e_n = C * U * (1.0 + n) if post else 0.0
    e = {"shift": 0.0 * du64, "scale": np.abs(du64) * np.abs(per("pre_w", 1.0)) * e_v}
    e["pre_b"], e["pre_w"] = 0.0 * du64, np.abs(du64 * (1.0 + per("scale", 0.0))) * e_v
    e3, e4 = e_d, e_d * n + d * e_n
    pw, pb = (np.abs(per("post_w", 1.0)), np.abs(per("post_b", 0.0))) if post else (1.0, 0.0)
    e["gate"] = np.abs(per("res_scale", 1.0)) * (pw * e4 + pb * e3)
    e["res_scale"] = np.abs(per("gate", 1.0)) * (pw * e4 + pb * e3)
    a = np.abs(per("gate", 1.0) * per("res_scale", 1.0))
    e["post_w"], e["post_b"] = a * e4, a * e3
    # the sums behind a gradient (S1 and S2, or S3 and S4) are rounded one by one before they are put together
    both = {"scale": np.abs(du64) * (np.abs(per("pre_w", 1.0) * k["xhat"]) + np.abs(per("pre_b", 0.0))),
            "gate": np.abs(per("res_scale", 1.0)) * d * (pw * n + pb), "res_scale": np.abs(per("gate", 1.0)) * d * (pw * n + pb)}
    rms_of = lambda t: float(np.sqrt(np.mean(np.square(t))))  # noqa: E731
    for name, got in grads.items():
        if not post and name.startswith("post"):
            continue
        axes = (1,) if got.dim() == 2 else (0, 1)
        size = np.maximum(mag[name], both[name].sum(axes) if name in both else 0.0)
        tol = e[name].sum(axes) + (128 + B) * U * size + 8 * U * np.abs(want[name])
        err = np.abs(got.cpu().double().numpy() - want[name])
        assert (err <= tol).all(), (name, float((err / tol).max()))
        # one row more or less is off by a part of 1 / rows of the size in every channel, above this for up to 2^19 rows
        assert rms_of(err) <= 32 * U * rms_of(size), (name, rms_of(err) / rms_of(size) / U)
