"""The steps of one block of sr_blocks8_fwd, each from what the call left in its scratch: the residual products and
their operands bit for bit from sr_quantize8 and sr_linear8, the LayerNorm codes through the products that they enter."""
import numpy as np
import pytest

import gpu_helpers as gh
from oracle import quant8 as oq
from oracle.block import gelu, ln_fwd
from oracle.numerics import storage_to_f64
from paper_2607_02829_amd import abi, device, inputs

pytestmark = pytest.mark.gpu


def _w(name, B, S, D, H, F, kind, dtype="bf16"):
    return inputs.small(name, B=B, Hg=1, Wg=S, D=D, H=H, F=F, kind=kind, dtype=dtype)


CASES = {}
for _kind in ("preln", "adaln"):
    # rows of the residual products from a few to those of the dense blocks at 0.25 deg: every tile that they are cut
    # into, with samples that end inside one
    CASES[f"16_rows_{_kind}"] = _w("s8_a", 2, 8, 1024, 16, 4096, _kind)
    CASES[f"128_rows_{_kind}"] = _w("s8_b", 2, 64, 1024, 16, 4096, _kind)
    CASES[f"1014_rows_{_kind}"] = _w("s8_c", 3, 338, 1024, 16, 4096, _kind)
    CASES[f"2026_rows_{_kind}"] = _w("s8_d", 2, 1013, 1024, 16, 4096, _kind)
    CASES[f"4026_rows_{_kind}"] = _w("s8_e", 2, 2013, 1024, 16, 4096, _kind)
    CASES[f"16200_rows_{_kind}"] = _w("s8_f", 2, 8100, 1024, 16, 4096, _kind)
    CASES[f"2026_rows_f32_{_kind}"] = _w("s8_g", 2, 1013, 1024, 16, 2048, _kind, "f32")
    CASES[f"4026_rows_f32_{_kind}"] = _w("s8_h", 2, 2013, 1024, 16, 2048, _kind, "f32")
    for _D, _H in ((64, 2), (512, 8), (576, 9), (1088, 17), (2048, 32)):   # rows of a LayerNorm
        CASES[f"D{_D}_{_kind}"] = _w("s8_i", 2, 45, _D, _H, 1024, _kind)
        CASES[f"D{_D}_f32_{_kind}"] = _w("s8_j", 2, 45, _D, _H, 1024, _kind, "f32")


def _layout(w):
    """Byte offset, shape and type of the buffers in the scratch, and its size."""
    M, D, F, e = w.B * w.L, w.D, w.F, 2 if w.dtype == "bf16" else 4
    t = "bfloat16" if w.dtype == "bf16" else "float32"
    parts = [("hin", (M, D), "float32", 4), ("h1", (M, D), "float32", 4), ("qkv", (M, 3 * D), t, e), ("O", (M, D), t, e),
             ("lse", (w.B * w.H, w.L), "float32", 4), ("gz", (M, F), t, e)]
    if w.kind == "adaln":
        parts.append(("mod", (w.B, 6 * D), "float32", 4))
    parts += [("codes", (M * max(D, F),), "int8", 1), ("scales", (M,), "float32", 4)]
    out, off = {}, 0
    for name, shape, dt, size in parts:
        off = (off + 255) & ~255
        out[name] = (off, shape, dt, size)
        off += int(np.prod(shape)) * size
    return out, off


@pytest.mark.parametrize("case", list(CASES))
def test_steps_of_a_block(case):
    import torch
    w = CASES[case]
    M, D, F = w.B * w.L, w.D, w.F
    ada = w.kind == "adaln"
    print(f"[blocks8 steps {case}] B={w.B} S={w.L} D={D} F={F} {w.dtype}", flush=True)
    h, params, cond, _ = gh.host_inputs(w, 1)
    cfg = device.config_for(w, n_blocks=1)
    dp = device.DeviceParams(params, w.kind)
    p8 = device.DeviceParams8(dp)
    p, t8 = dp.tensors[0], p8.tensors[0]
    hd = device.to_device(h)
    places, size = _layout(w)
    n = abi.sr_blocks8_scratch_bytes(cfg, w.L)
    assert n == size
    buf, out = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), torch.empty_like(hd)
    abi.sr_blocks8_fwd(cfg, w.L, p8.array, device.to_device(cond) if ada else None, hd, out, buf)
    torch.cuda.synchronize()
    s = {k: buf[o:o + int(np.prod(sh)) * b].view(getattr(torch, dt)).view(sh) for k, (o, sh, dt, b) in places.items()}
    dt = abi.SR_BF16 if w.dtype == "bf16" else abi.SR_F32
    h0 = hd.float().view(M, D)

    def rows(x):
        q, sc = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
        abi.sr_quantize8(abi.SR_Q8_ROW, dt, M, x.shape[1], x, q, sc)
        return q, sc

    def branch(q, sc, name, resid, gate_at):
        """resid + gate (product): the values it may have, with the multiplication rounded or fused into the sum."""
        v = torch.empty((M, D), device="cuda")
        abi.sr_linear8(abi.SR_F32, abi.SR_ACT_NONE, M, D, q.shape[1], q, sc, t8["w_" + name], t8["s_" + name],
                       p["b_" + name].float(), v)
        if not ada:
            return resid + v, resid + v
        g = s["mod"][:, gate_at:gate_at + D].repeat_interleave(w.L, 0)
        return resid + v * g, (resid.double() + v.double() * g.double()).float()

    def equal(got, either):
        return bool(((got == either[0]) | (got == either[1])).all())

    # output projection, and the second MLP product, whose codes are still there
    assert equal(s["h1"], branch(*rows(s["O"]), "o", h0, 2 * D))
    q, sc = rows(s["gz"])
    assert torch.equal(q.view(-1), s["codes"][:M * F]) and torch.equal(sc, s["scales"])
    assert equal(s["hin"], branch(q, sc, "fc2", s["h1"], 5 * D))
    assert torch.equal(out.view(M, D), s["hin"].to(out.dtype))

    # The LayerNorms' codes, on some rows: of a LayerNorm in fp32 (2e-6 of the largest value at most) a code differs from
    # the oracle's where 127 x / a lies within 2.5e-4 of a tie, one in 2000, by a step, against the 0.29 steps in the mean
    # square that rounding costs every code: 0.08 of what the codes of tokens and weights change in the product, and
    # bf16's own rounding of that, 2^-8 / sqrt(12) of the result, is a tenth of their 1 %.
    r = np.unique(np.linspace(0, M - 1, 96).astype(int))
    rt = torch.from_numpy(r).cuda()
    mod = s["mod"].double().cpu().numpy() if ada else None
    p64 = {k: storage_to_f64(v) for k, v in params[0].items()}

    def norm(x, k, at):
        x = x[rt].double().cpu().numpy()
        if ada:
            m = mod[r // w.L]
            return ln_fwd(x, None, None, 1e-6)[0] * (1.0 + m[:, at + D:at + 2 * D]) + m[:, at:at + D]
        return ln_fwd(x, p64[f"ln{k}_w"], p64[f"ln{k}_b"], 1e-6)[0]

    for k, x, at, name, got in (("1", h0, 0, "qkv", "qkv"), ("2", s["h1"], 3 * D, "fc1", "gz")):
        u = norm(x, k, at)
        full = u @ p64["w_" + name].T + p64["b_" + name]
        codes = oq.linear(*oq.quant_rows(u), t8["w_" + name].cpu().numpy(), t8["s_" + name].cpu().numpy(), p64["b_" + name])
        if name == "fc1":
            full, codes = gelu(full), gelu(codes)
        y = s[got][rt].double().cpu().numpy()
        err, eight = np.linalg.norm(y - codes), np.linalg.norm(codes - full)
        assert err <= (0.25 if w.dtype == "bf16" else 0.15) * eight, (name, err, eight)
