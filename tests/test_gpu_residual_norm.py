"""sr_residual_norm_fwd / _bwd against their 64-bit form.

Tolerances, u = 2^-24.  A row's mean and mean square are sums of at most 8192 values, at most 16 in a lane one
after another and 13 levels above: 29 roundings each, so Norm(z) is off by at most 32 u (1 + |mean| rstd) + 34 u |Norm(z)|
with the products; what follows adds at most 8 roundings of the summands' magnitudes.  With the inputs here (|mean| rstd < 4)
that is C u = 256 u of the row's largest magnitudes, plus half a step of the result's type.  A column sum over n rows
in any order is off by at most n u of its summands' magnitudes, its summands by C u of the row's."""
import numpy as np
import pytest

from oracle import block_ops as ob
from paper_2607_02829_amd import abi

pytestmark = pytest.mark.gpu

U, C = 2.0 ** -24, 256.0
EPS = 1e-6

CASES = [
    # B, S, D, rms, post, names of the parameters, p, group, dtype, stream
    (1, 1, 1024, False, True, "post_w post_b res_scale pre_w pre_b", 0.0, 0, "bf16", "f32"),
    (1, 1, 1, True, True, "post_w res_scale pre_w", 0.0, 0, "f32", "f32"),
    (2, 3, 1, False, True, "pre_w pre_b gate", 0.0, 0, "f32", "f32"),
    (2, 5, 7, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.3, 0, "bf16", "bf16"),
    (3, 50, 64, True, True, "gate shift scale", 0.1, 0, "bf16", "f32"),
    (1, 130, 129, False, False, "res_scale pre_w", 0.2, 1, "bf16", "f32"),
    (4, 33, 200, True, False, "", 0.0, 0, "bf16", "bf16"),
    (2, 70, 256, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.25, 0, "f32", "f32"),
    (2, 19, 511, True, True, "post_w post_b pre_w pre_b", 0.5, 0, "f32", "f32"),
    (5, 40, 512, False, True, "gate", 0.2, 40, "bf16", "f32"),
    (2, 300, 1024, False, True, "res_scale gate shift scale", 0.1, 0, "bf16", "f32"),
    (1, 100, 1024, True, True, "post_w res_scale pre_w", 0.0, 0, "bf16", "bf16"),
    (3, 7, 1027, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.1, 0, "bf16", "f32"),
    (2, 9, 2048, True, True, "post_w gate scale", 0.0, 0, "f32", "f32"),
    (2, 9, 4000, False, False, "res_scale pre_w pre_b", 0.1, 0, "bf16", "f32"),
    (1, 5, 8192, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.1, 0, "bf16", "f32"),
    (1, 3, 8191, True, True, "post_w pre_w", 0.0, 0, "f32", "f32"),
    (2, 40, 2, False, True, "post_w res_scale gate shift scale", 0.2, 0, "bf16", "f32"),
    (1, 33, 3, True, True, "post_w post_b pre_w pre_b", 0.2, 0, "f32", "f32"),
    (3, 21, 5, False, False, "res_scale gate", 0.2, 0, "bf16", "bf16"),
    (2, 25, 30, True, True, "post_w pre_w scale", 0.1, 0, "bf16", "f32"),
    (1, 90, 770, False, True, "post_w post_b res_scale pre_w pre_b", 0.1, 0, "bf16", "f32"),
    (2, 30, 1536, True, True, "post_w pre_w gate", 0.0, 0, "f32", "f32"),
    (1, 20, 2999, False, True, "res_scale shift scale", 0.1, 0, "bf16", "bf16"),
    (1, 7, 5001, True, True, "post_w pre_w", 0.1, 0, "bf16", "f32"),
    (1, 9000, 64, False, True, "post_w post_b gate", 0.1, 0, "bf16", "f32"),             # results past the caches
    (1200, 2, 32, False, True, "res_scale gate shift scale", 0.1, 2, "bf16", "f32"),     # more samples than workgroups
]


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _sr(name):
    return abi.SR_BF16 if name == "bf16" else abi.SR_F32


def _setup(c, seed=1, mod_extra=3):
    import torch
    B, S, D, rms, post, names, p, group, dtype, stream = c
    g = torch.Generator().manual_seed(seed + D + S)
    dt, st = _dt(dtype), _dt(stream)
    x = (2 * torch.randn((B, S, D), generator=g) + 0.7).to(st)
    y = (torch.randn((B, S, D), generator=g) * torch.exp(torch.randn((B, S, 1), generator=g)) - 0.3).to(dt)
    w, stride = {}, D + mod_extra
    for n in names.split():
        if n in ("gate", "shift", "scale"):
            w[n] = (0.5 * torch.randn((B, stride), generator=g))
        else:
            w[n] = ((1.0 if n.endswith("_w") else 0.0) + 0.3 * torch.randn(D, generator=g)).to(dt)
    cfg = abi.SrResidualNorm(B=B, S=S, D=D, dtype=_sr(dtype), stream_dtype=_sr(stream),
                             norm=abi.SR_NORM_RMS if rms else abi.SR_NORM_LAYER, post=int(post), eps=EPS, mod_stride=stride,
                             drop=abi.SrDrop(p=p, seed=9, step=2, group=group, first_row=5))
    keep = ob.drop_keep(B * S, D, p, 9, 2, 5, group).reshape(B, S, D) if p > 0 else None
    dev = {k: v.cuda() for k, v in w.items()}
    w64 = {k: (v[:, :D] if v.dim() == 2 else v).double().numpy() for k, v in w.items()}
    return cfg, x, y, dev, w64, keep, g


def _near(got, want, scale, what, eps=0.0):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    tol = eps * np.abs(want) + C * U * scale
    err = np.abs(got - want)
    assert np.isfinite(got).all() and (err <= tol).all(), (what, float((err / np.maximum(tol, 1e-300)).max()))


def _rowmax(*ts):
    return sum(np.abs(t).max(-1, keepdims=True) for t in ts) + 1e-30


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", "_"))
def test_forward_and_backward(c):
    import torch
    B, S, D, rms, post, names, p, group, dtype, stream = c
    cfg, x, y, w, w64, keep, g = _setup(c)
    dt, st, M = _dt(dtype), _dt(stream), B * S
    e, es = torch.finfo(dt).eps / 2, torch.finfo(st).eps / 2
    f = ob.drop_factor(p)
    params = abi.residual_norm_params(**w)
    xd, yd = x.cuda(), y.cuda()
    x1 = torch.full((M * D + 8,), 3.5, dtype=st, device="cuda")
    u = torch.full((M * D + 8,), 3.5, dtype=dt, device="cuda")
    stats = torch.full((4 * M + 4,), 3.5, device="cuda")
    abi.sr_residual_norm_fwd(cfg, params, xd, yd, x1, u, stats=stats)
    for t in (x1[M * D:], u[M * D:], stats[4 * M:]):
        assert (t == 3.5).all()
    got1 = x1[:M * D].view(B, S, D).cpu()
    x64, y64 = x.double().numpy(), y.double().numpy()
    # the second norm reads the stored x1: checked on what the kernel stored
    want1, want_u, k = ob.residual_norm(x64, y64, w64, rms, post, EPS, keep, f, stored=lambda _: got1.double().numpy())
    n_mag = np.abs(want1 - x64)
    _near(got1.double(), want1, _rowmax(x64, n_mag, 1.0 + np.abs(np.broadcast_to(
        np.asarray(w64.get("gate", np.ones((B, D)))[:, None, :] * w64.get("res_scale", 1.0)), x64.shape)) * f * 8), "x1", es)
    _near(u[:M * D].view(B, S, D).cpu().double(), want_u, _rowmax(want_u, k["t"] * (1 + np.abs(w64.get("scale", np.zeros((B, D)))[:, None, :]))) + 8,
          "u", e)

    dx1 = (0.3 * torch.randn((B, S, D), generator=g)).to(st)
    du = (0.3 * torch.randn((B, S, D), generator=g)).to(dt)
    grads = {n: torch.full((v.shape[0], D) if v.dim() == 2 else (D,), 9.0, device="cuda") for n, v in w.items()}
    dx = torch.full((M * D + 8,), 3.5, dtype=st, device="cuda")
    dy = torch.full((M * D + 8,), 3.5, dtype=dt, device="cuda")
    scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    abi.sr_residual_norm_bwd(cfg, params, x1, yd, stats, dx1.cuda(), du.cuda(), dx, dy, abi.residual_norm_grads(**grads), scratch)
    for t in (dx[M * D:], dy[M * D:]):
        assert (t == 3.5).all()
    wdx, wdy, wg, mag = ob.residual_norm_bwd(k, dx1.double().numpy(), du.double().numpy())
    big = lambda n, lo: 1.0 + np.abs(w64.get(n, np.zeros(1))).max() if lo else np.abs(w64.get(n, np.ones(1))).max()  # noqa: E731
    du_mag = _rowmax(du.double().numpy()) * big("scale", True) * max(1.0, big("pre_w", False))
    dx_mag = _rowmax(dx1.double().numpy()) + k["xrstd"] * du_mag * (1 + _rowmax(k["xhat"]))
    _near(dx[:M * D].view(B, S, D).cpu().double(), wdx, dx_mag, "dx", es)
    a_mag = big("gate", False) * big("res_scale", False) * f
    dy_mag = dx_mag * a_mag * max(1.0, big("post_w", False)) * (k["yrstd"] * (1 + _rowmax(k["yhat"])) if post else 1.0)
    _near(dy[:M * D].view(B, S, D).cpu().double(), wdy, dy_mag, "dy", e)
    # what a summand can be off by, over the rows, and the sum's own roundings
    hat = _rowmax(k["xhat"]).max()
    n_max = np.abs(k["n"]).max() + 1.0
    for n, got in grads.items():
        rows = S if got.dim() == 2 else M
        if n in ("shift", "scale", "pre_w", "pre_b"):
            per_row = du_mag.max() * (1 + hat) * max(1.0, big("pre_w", False)) * (1 + big("pre_b", True))
        else:
            per_row = dx_mag.max() * max(1.0, big("gate", False)) * max(1.0, big("res_scale", False)) * f * (n_max + _rowmax(k.get("yhat", np.zeros(1))).max())
        if not post and n.startswith("post"):
            assert (got == 0).all()
            continue
        tol = rows * U * mag[n] + C * U * per_row * rows
        err = np.abs(got.cpu().double().numpy() - wg[n])
        assert (err <= tol).all(), (n, float((err / tol).max()))


def test_in_place_and_repeatable():
    import torch
    c = (3, 40, 320, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.2, 0, "bf16", "f32")
    cfg, x, y, w, _, _, g = _setup(c)
    B, S, D, M = 3, 40, 320, 120
    params = abi.residual_norm_params(**w)
    res = []
    for inplace in (False, True, True):
        xd, yd = x.cuda(), y.cuda()
        x1 = xd if inplace else torch.empty_like(xd)
        u, stats = torch.empty_like(yd), torch.empty((4, M), device="cuda")
        abi.sr_residual_norm_fwd(cfg, params, xd, yd, x1, u, stats=stats)
        dx1 = (0.3 * x).cuda()
        dx = dx1 if inplace else torch.empty_like(dx1)
        dy = torch.empty_like(yd)
        grads = {n: torch.empty((B, D) if v.dim() == 2 else (D,), device="cuda") for n, v in w.items()}
        scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
        abi.sr_residual_norm_bwd(cfg, params, x1, yd, stats, dx1, u, dx, dy, abi.residual_norm_grads(**grads), scratch)
        res.append([x1, u, stats, dx, dy, *grads.values()])
    for other in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(res[0], other))


def test_parts_of_the_step():
    # the norm before a first branch (no y), the sum after a last one (no u), one gradient only
    import torch
    c = (2, 30, 192, False, True, "post_w post_b res_scale pre_w pre_b gate shift scale", 0.1, 0, "f32", "f32")
    cfg, x, y, w, w64, keep, g = _setup(c)
    B, S, D, M = 2, 30, 192, 60
    params = abi.residual_norm_params(**w)
    xd, yd = x.cuda(), y.cuda()
    full = dict(x1=torch.empty_like(xd), u=torch.empty_like(yd), stats=torch.empty((4, M), device="cuda"))
    abi.sr_residual_norm_fwd(cfg, params, xd, yd, full["x1"], full["u"], stats=full["stats"])
    x1, st = torch.empty_like(xd), torch.full((4, M), 2.5, device="cuda")
    abi.sr_residual_norm_fwd(cfg, params, xd, yd, x1, None, stats=st)
    assert torch.equal(x1, full["x1"]) and torch.equal(st[:2], full["stats"][:2]) and (st[2:] == 2.5).all()
    u, st = torch.empty_like(yd), torch.full((4, M), 2.5, device="cuda")
    abi.sr_residual_norm_fwd(cfg, params, x1, None, None, u, stats=st)
    assert torch.equal(u, full["u"]) and torch.equal(st[2:], full["stats"][2:]) and (st[:2] == 2.5).all()

    dx1, du = torch.randn((B, S, D), generator=g), torch.randn((B, S, D), generator=g)
    scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    none = abi.residual_norm_grads()

    def bwd(y=yd, dx1=dx1.cuda(), du=du.cuda(), grads=none):
        dx, dy = torch.empty_like(xd), None if y is None else torch.empty_like(yd)
        abi.sr_residual_norm_bwd(cfg, params, full["x1"], y, full["stats"], dx1, du, dx, dy, grads, scratch)
        return dx, dy

    dx, dy = bwd()
    dxa, _ = bwd(y=None)
    assert torch.equal(dx, dxa)
    only_u, only_x = bwd(dx1=None), bwd(du=None)
    assert torch.equal(only_x[0].cpu(), dx1)
    # linear in (dx1, du): both roundings of dx, one more of the sum
    for a, b, t in zip(only_u, only_x, (dx, dy)):
        assert (a + b - t).abs().max() <= 2.0 ** -20 * (a.abs() + b.abs()).max()
    # gradients of parameters that no branch reads are zeros
    g2 = {n: torch.full((B, D) if w[n].dim() == 2 else (D,), 7.0, device="cuda") for n in w}
    bwd(y=None, grads=abi.residual_norm_grads(**g2))
    assert all((g2[n] == 0).all() for n in ("post_w", "post_b", "res_scale", "gate"))
    bwd(du=None, grads=abi.residual_norm_grads(**g2))
    assert all((g2[n] == 0).all() for n in ("pre_w", "pre_b", "shift", "scale"))


def test_dropped_nan_and_other_rows():
    # a NaN that is dropped does not count (without a norm before it); a row's NaN stays in the row
    import torch
    B, S, D = 1, 24, 96
    cfg = abi.SrResidualNorm(B=B, S=S, D=D, dtype=abi.SR_F32, stream_dtype=abi.SR_F32, norm=abi.SR_NORM_RMS, post=0, eps=EPS,
                             mod_stride=D, drop=abi.SrDrop(p=0.5, seed=3, step=3))
    keep = torch.from_numpy(ob.drop_keep(S, D, 0.5, 3, 3))
    g = torch.Generator().manual_seed(1)
    x, y = torch.randn((S, D), generator=g), torch.randn((S, D), generator=g)
    bad = torch.where(keep, y, float("nan")).cuda()
    rs = torch.randn(D, generator=g).cuda()
    params = abi.residual_norm_params(res_scale=rs)
    scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    out = []
    for yy in (y.cuda(), bad):
        x1, u, st = torch.empty((S, D), device="cuda"), torch.empty((S, D), device="cuda"), torch.empty((4, S), device="cuda")
        abi.sr_residual_norm_fwd(cfg, params, x.cuda(), yy, x1, u, stats=st)
        dx, dy, drs = torch.empty_like(x1), torch.empty_like(x1), torch.empty(D, device="cuda")
        abi.sr_residual_norm_bwd(cfg, params, x1, yy, st, u, u, dx, dy, abi.residual_norm_grads(res_scale=drs), scratch)
        out.append((x1, u, dx, dy, drs))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    y2 = y.clone()
    y2[7, 3], x2 = float("nan"), x.clone()
    x2[9, 0] = float("inf")
    x1, u = torch.empty((S, D), device="cuda"), torch.empty((S, D), device="cuda")
    cfg.post, cfg.drop.p = 1, 0.0
    abi.sr_residual_norm_fwd(cfg, params, x2.cuda(), y2.cuda(), x1, u)
    rows = torch.isfinite(u).all(1).cpu()
    assert rows.sum() == S - 2 and not rows[7] and not rows[9]


def test_codes_straight_from_the_norm():
    import torch
    for D, rms in ((64, False), (128, True), (200, False), (1024, False), (1100, True), (4096, True), (1, True), (3, False), (129, False), (255, True), (1022, True)):
        c = (2, 21, D, rms, True, "post_w res_scale pre_w shift scale", 0.1, 0, "bf16", "f32")
        cfg, x, y, w, w64, keep, _ = _setup(c, mod_extra=4 - D % 4)
        M = 42
        q, e, _, _ = abi.f8_buffers(M, D)
        q.fill_(0xEE)
        e.fill_(0xEE)
        x1, x1b, u = torch.empty((M, D), device="cuda"), torch.empty((M, D), device="cuda"), torch.empty((M, D), device="cuda")
        params = abi.residual_norm_params(**w)
        ub = torch.empty((M, D), dtype=torch.bfloat16, device="cuda")
        abi.sr_residual_norm_fwd(cfg, params, x.cuda(), y.cuda(), x1, ub, q, e)
        # the fp32 mode of the same values gives u before its rounding
        c32 = abi.SrResidualNorm.from_buffer_copy(cfg)
        c32.dtype = abi.SR_F32
        w32 = {k: v.float() for k, v in w.items()}
        abi.sr_residual_norm_fwd(c32, abi.residual_norm_params(**w32), x.cuda(), y.float().cuda(), x1b, u)
        assert torch.equal(x1, x1b) and torch.equal(u.bfloat16(), ub)
        wq, we, _ = ob.f8_quantize(u.cpu().double().numpy())
        assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(e.cpu().numpy()[:, :M], we)
        assert (e[:, M:] == 0xEE).all()


@pytest.mark.parametrize("D", [257, 300, 512, 513, 700, 1000, 1024, 1025, 1536, 1537, 2047, 2048])
@pytest.mark.parametrize("rms,dtype", [(False, "bf16"), (True, "f32")])
def test_a_row_does_not_depend_on_how_many_there_are(D, rms, dtype):
    # 40 rows are taken by wider teams than 600; their results are those rows' of the larger call, bit for bit
    import torch
    c = (1, 600, D, rms, True, "post_w post_b res_scale pre_w pre_b", 0.1, 0, dtype, "f32")
    cfg, x, y, w, _, _, g = _setup(c, mod_extra=0)
    dt = _dt(dtype)
    dx1, du = torch.randn((600, D), generator=g).cuda(), torch.randn((600, D), generator=g).to(dt).cuda()
    xd, yd, first = x.view(600, D).cuda(), y.view(600, D).cuda(), cfg.drop.first_row
    params = abi.residual_norm_params(**w)
    out = []
    for lo, hi in ((0, 600), (560, 600)):
        n = hi - lo
        cfg.S, cfg.drop.first_row = n, first + lo
        x1, u, st = torch.empty((n, D), device="cuda"), torch.empty((n, D), dtype=dt, device="cuda"), torch.empty((4, n), device="cuda")
        dx, dy = torch.empty((n, D), device="cuda"), torch.empty((n, D), dtype=dt, device="cuda")
        a = [t[lo:hi].clone() for t in (xd, yd, dx1, du)]
        abi.sr_residual_norm_fwd(cfg, params, a[0], a[1], x1, u, None, None, st)
        scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
        abi.sr_residual_norm_bwd(cfg, params, x1, a[1], st, a[2], a[3], dx, dy, abi.residual_norm_grads(), scratch)
        out.append((x1, u, dx, dy, st.T))
    for p, q in zip(*out):
        assert torch.equal(p[560:], q)


def test_many_calls_of_few_rows_agree():
    # waves of one workgroup share their SIMDs here: every wave draws its own words, in every call
    import torch
    for D in (1100, 1500, 2048):
        c = (2, 21, D, False, True, "post_w res_scale", 0.1, 0, "f32", "f32")
        cfg, x, y, w, w64, keep, _ = _setup(c, mod_extra=0)
        params, xd, yd = abi.residual_norm_params(**w), x.cuda(), y.cuda()
        n = (42 * D + 3) // 4 * 4
        x1, u = torch.zeros((300, n), device="cuda"), torch.zeros((300, n), device="cuda")
        for i in range(300):
            abi.sr_residual_norm_fwd(cfg, params, xd, yd, x1[i], u[i])
        assert bool((x1 == x1[0]).all()) and bool((u == u[0]).all())
        moved = (x1[0, :42 * D].view(2, 21, D).cpu() != x).numpy()
        assert np.array_equal(moved & ~keep, np.zeros_like(keep)) and moved.mean() > 0.8
