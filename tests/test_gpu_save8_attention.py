"""SR_BLOCK_SAVE8 with peaked attention: the backward's probabilities sum to one over the keys, whatever the
size of the logits, so its gradients are those of a softmax."""
import numpy as np
import pytest

import gpu_helpers as gh
from oracle import quant8 as oq
from oracle import stack as ostack
from oracle.numerics import f32_to_storage, storage_to_f32, storage_to_f64
from paper_2607_02829_amd import abi, device, inputs

pytestmark = pytest.mark.gpu

CASES = {
    "bf16": inputs.small("pk_p", B=2, Hg=9, Wg=15, D=256, H=4, F=512),
    "f32": inputs.small("pk_f", B=1, Hg=7, Wg=11, D=128, H=2, F=256, dtype="f32"),
    "adaln_bf16": inputs.small("pk_a", B=2, Hg=9, Wg=15, D=256, H=4, F=512, kind="adaln"),
    "head_dim_32": inputs.small("pk_3", B=2, Hg=9, Wg=13, D=128, H=4, F=256),
    "head_dim_128": inputs.small("pk_h", B=1, Hg=10, Wg=13, D=256, H=2, F=512),
    "few_heads_long": inputs.small("pk_l", B=1, Hg=25, Wg=41, D=128, H=2, F=256),
}


def peaked(w, target):
    """One block's inputs with the q and k rows scaled by a power of two, so that the logits deviate by about target."""
    h, params, cond, dh = gh.host_inputs(w, 1)
    c64 = storage_to_f64(cond) if cond is not None else None

    def caches():
        return ostack.stack_fwd(storage_to_f64(h), ostack.params_f64(params), w.H, 1e-6, w.kind, c64)[1]

    def logits(c):
        return c["q"] @ c["k"].swapaxes(-1, -2) / np.sqrt(w.D // w.H)

    f = np.float32(2.0 ** np.round(np.log2(np.sqrt(target / logits(caches()[0]).std()))))
    for n in ("w_qkv", "b_qkv"):
        t = storage_to_f32(params[0][n]).copy()
        t[:2 * w.D] *= f
        params[0][n] = f32_to_storage(t, params[0][n])
    c = caches()
    return h, params, cond, dh, c, logits(c[0])


def run(w, h, params, cond, dh, drop=()):
    import torch
    cfg = device.config_for(w, n_blocks=1)
    cfg.kind |= abi.SR_BLOCK_SAVE8
    dp = device.DeviceParams(params, w.kind)
    hd, dhd = device.to_device(h), device.to_device(dh)
    c = device.to_device(cond) if cond is not None else None
    out, dx = torch.empty_like(hd), torch.empty_like(dhd)
    saved, scratch = device.workspace(cfg, w.L)
    saved.fill_(0xFF)
    scratch.fill_(0xFF)
    g = device.DeviceGrads(w, 1)
    for n in drop:
        setattr(g.array[0], n, None)
    abi.sr_sparse_blocks_fwd(cfg, w.L, dp.array, c, hd, out, saved, scratch)
    abi.sr_sparse_blocks_bwd(cfg, w.L, dp.array, c, saved, dhd, dx, g.array, None, scratch)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in g.tensors[0].items()}, device.to_host(dx)


@pytest.mark.parametrize("target", [4.0, 16.0, 64.0])
@pytest.mark.parametrize("case", list(CASES))
def test_probabilities_sum_to_one(case, target, monkeypatch):
    w = CASES[case]
    D, scale = w.D, 1.0 / np.sqrt(w.D // w.H)
    print(f"[save8 peaked {case}] logits of {target}, S={w.L} D={D} {w.dtype} {w.kind}", flush=True)
    h, params, cond, dh, caches, s = peaked(w, target)
    g, _ = run(w, h, params, cond, dh)
    # sizes of what is summed, from the oracle's backward of the kept values
    rec = []
    inner = oq._kept_attention_bwd
    monkeypatch.setattr(oq, "_kept_attention_bwd", lambda *a: rec.append((a, inner(*a))) or rec[-1][1])
    p64 = ostack.params_f64(params)
    oq.stack_bwd_kept(storage_to_f64(dh), p64, caches)
    (args, (dq, dk, dv)), = rec
    q, k, v, dO = args[0], args[1], args[2], args[-1]
    P = np.exp(q @ k.swapaxes(-1, -2) * scale)
    P /= P.sum(-1, keepdims=True)
    PdP, O = P * (dO @ v.swapaxes(-1, -2)), P @ v
    dS = PdP - P * (dO * O).sum(-1, keepdims=True)
    sq = lambda t: float((t * t).sum())  # noqa: E731
    # Rounded on the way, each by at most u of itself and independently: dO, P (dv sums over both), dv;  P and O (in
    # delta), dS, dk.  The exponents, of logits up to max |s|, are off by a few of its steps: that is the other part.
    u = (2.0 ** -8 if w.dtype == "bf16" else 2.0 ** -24) + 8 * np.abs(s).max() * 2.0 ** -24
    # v: with rows of P that sum to one, sum_j dv_j = sum_i dO_i = (sum_i da_i) W_o
    want = g["b_o"].astype(np.float64) @ p64[0]["w_o"]
    err = np.linalg.norm(g["b_qkv"][2 * D:] - want)
    assert err <= u * np.sqrt(2 * sq(dO) + sq(dv)), (err, np.linalg.norm(want))
    # k: rows of dS sum to zero, so a shift of every key changes nothing
    rows = (dS * dS + PdP * PdP).sum(-1) + (dO * dO * O * O).sum(-1)
    err = np.linalg.norm(g["b_qkv"][D:2 * D])
    assert err <= u * np.sqrt(scale * scale * float(((q * q).sum(-1) * rows).sum()) + sq(dk)), err


def test_output_projection_gradients_one_at_a_time():
    w = CASES["bf16"]
    h, params, cond, dh, _, _ = peaked(w, 4.0)
    both, dx = run(w, h, params, cond, dh)
    for drop, kept in (("w_o", "b_o"), ("b_o", "w_o")):
        one, dx1 = run(w, h, params, cond, dh, drop=(drop,))
        assert np.array_equal(one[kept], both[kept]) and np.array_equal(dx1, dx)
