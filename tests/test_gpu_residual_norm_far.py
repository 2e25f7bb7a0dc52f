"""sr_residual_norm_fwd / _bwd with as many rows as they take: numbers of rows whose sums pass 2^31."""
import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.gpu

PERIOD, GUARD = 1 << 16, 1 << 12


def _rows(n, dtype, seed):
    """n values, the same again after every PERIOD, between two guards."""
    import torch
    t = torch.full((GUARD + n + GUARD,), 99.0, dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    first = torch.randn(PERIOD, generator=g, device="cuda").to(dtype)
    body = t[GUARD:GUARD + n]
    whole = n // PERIOD * PERIOD
    body[:whole].view(-1, PERIOD).copy_(first.expand(whole // PERIOD, PERIOD))
    body[whole:] = first[:n - whole]
    return t, body


def _periodic(t, n):
    """Every period of the result is the first one, and the guards are as they were."""
    import torch
    body, whole = t[GUARD:GUARD + n], n // PERIOD * PERIOD
    assert bool((t[:GUARD] == 99.0).all()) and bool((t[GUARD + n:] == 99.0).all())
    first = body[:PERIOD]
    for at in range(0, whole, 1 << 28):   # in pieces: the comparison makes a tensor of its own
        piece = body[at:min(at + (1 << 28), whole)].view(-1, PERIOD)
        assert bool((piece == first).all()), at
    assert torch.equal(body[whole:], first[:n - whole])


@pytest.mark.parametrize("S", [(1 << 31) - 1023, (1 << 31) - 1])
def test_one_sample_of_nearly_2_31_rows(S):
    # one channel and no mean: every row is a function of its own two values, so the rows repeat as the inputs do
    import torch
    print(f"[residual norm far] {S} rows", flush=True)
    cfg = abi.SrResidualNorm(B=1, S=S, D=1, dtype=abi.SR_BF16, stream_dtype=abi.SR_BF16, norm=abi.SR_NORM_RMS, post=1, eps=0.5,
                             mod_stride=0)
    w = {k: torch.full((8,), v, dtype=torch.bfloat16, device="cuda") for k, v in (("post_w", 1.5), ("pre_w", -0.75))}
    params = abi.residual_norm_params(**w)
    (_, x), (_, y) = _rows(S, torch.bfloat16, 1), _rows(S, torch.bfloat16, 2)
    out = {n: torch.full((GUARD + S + GUARD,), 99.0, dtype=torch.bfloat16, device="cuda") for n in ("x1", "u", "dx", "dy")}
    body = {n: t[GUARD:GUARD + S] for n, t in out.items()}
    stats = torch.empty((4 * S + 4,), device="cuda")
    abi.sr_residual_norm_fwd(cfg, params, x, y, body["x1"], body["u"], stats=stats)
    torch.cuda.synchronize()
    print("forward done", flush=True)
    grads = {k: torch.full((4,), 99.0, device="cuda") for k in w}
    scratch = torch.empty(abi.sr_residual_norm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    abi.sr_residual_norm_bwd(cfg, params, body["x1"], y, stats, x, y, body["dx"], body["dy"], abi.residual_norm_grads(**grads),
                             scratch)
    torch.cuda.synchronize()
    print("backward done", flush=True)
    for n in out:
        _periodic(out[n], S)
    # the first period against the formulas, half a step of bf16 (2^-8 of the value) and fp32 besides
    x64, y64 = x[:PERIOD].double(), y[:PERIOD].double()
    x1 = x64 + 1.5 * y64 / torch.sqrt(y64 * y64 + 0.5)
    got = body["x1"][:PERIOD].double()
    assert bool(((got - x1).abs() <= 2.0 ** -8 * x1.abs() + 1e-5).all())
    u = -0.75 * got / torch.sqrt(got * got + 0.5)
    assert bool(((body["u"][:PERIOD].double() - u).abs() <= 2.0 ** -8 * u.abs() + 1e-5).all())
    del x, y, out, body, stats, scratch
    torch.cuda.empty_cache()
