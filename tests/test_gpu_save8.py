"""Blocks whose forward keeps its activations in 8 bits (SR_BLOCK_SAVE8): outputs bit for bit those without
it, gradients those of the kept values, and what changes in memory, routing, graphs and the trunk."""
import numpy as np
import pytest

import gpu_helpers as gh
from oracle import quant8 as oq
from oracle import stack as ostack
from oracle.numerics import storage_to_f64
from paper_2607_02829_amd import abi, device, inputs
from paper_2607_02829_amd.trunk import Trunk

pytestmark = pytest.mark.gpu


def _run(w, S, h, params, cond, dh, save8, scratch_fill=None):
    import torch
    nb = len(params)
    cfg = device.config_for(w, n_blocks=nb)
    if save8:
        cfg.kind |= abi.SR_BLOCK_SAVE8
    dp = device.DeviceParams(params, w.kind)
    hd, dhd = device.to_device(h), device.to_device(dh)
    c = device.to_device(cond) if cond is not None else None
    out, dx = torch.empty_like(hd), torch.empty_like(dhd)
    saved, scratch = device.workspace(cfg, S)
    guard = torch.full((saved.numel() + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    saved = guard[:saved.numel()]
    if scratch_fill is not None:
        scratch.fill_(scratch_fill)
    g = device.DeviceGrads(w, nb)
    dcond = torch.empty((w.B, w.D), dtype=torch.float32, device="cuda") if cond is not None else None
    abi.sr_sparse_blocks_fwd(cfg, S, dp.array, c, hd, out, saved, scratch)
    abi.sr_sparse_blocks_bwd(cfg, S, dp.array, c, saved, dhd, dx, g.array, dcond, scratch)
    torch.cuda.synchronize()
    assert bool((guard[saved.numel():] == 0x5A).all())
    res = {"h_out": device.to_host(out), "dh_in": device.to_host(dx),
           "grads": [{k: v.cpu().numpy() for k, v in gg.items()} for gg in g.tensors],
           "dcond": dcond.cpu().numpy() if dcond is not None else None}
    return res, saved.numel()


CASES = {
    "preln_bf16": (inputs.small("save8_p", B=2, Hg=9, Wg=15, D=256, H=4, F=1024), 2),
    "preln_f32": (inputs.small("save8_f", B=1, Hg=7, Wg=11, D=128, H=2, F=512, dtype="f32"), 2),
    "adaln_bf16": (inputs.small("save8_a", B=2, Hg=9, Wg=15, D=256, H=4, F=1024, kind="adaln"), 2),
    "adaln_f32": (inputs.small("save8_b", B=2, Hg=5, Wg=7, D=64, H=2, F=256, dtype="f32", kind="adaln"), 2),
    "head_dim_128": (inputs.small("save8_h", B=1, Hg=10, Wg=13, D=256, H=2, F=512), 1),
    "one_token": (inputs.small("save8_1", B=3, Hg=1, Wg=1, D=128, H=2, F=256), 2),
    "three_blocks": (inputs.small("save8_3", B=1, Hg=16, Wg=33, D=512, H=8, F=1024), 3),
}


@pytest.mark.parametrize("case", list(CASES))
def test_gradients_are_those_of_the_kept_values(case):
    w, nb = CASES[case]
    S = w.L
    print(f"[save8 {case}] B={w.B} S={S} D={w.D} {w.dtype} {w.kind}", flush=True)
    h, params, cond, dh = gh.host_inputs(w, nb)
    got, _ = _run(w, S, h, params, cond, dh, True)
    plain, _ = _run(w, S, h, params, cond, dh, False)
    assert np.array_equal(got["h_out"], plain["h_out"])
    p64 = ostack.params_f64(params)
    c64 = storage_to_f64(cond) if cond is not None else None
    h_out, caches = ostack.stack_fwd(storage_to_f64(h), p64, w.H, 1e-6, w.kind, c64)
    dh_in, grads, dcond = oq.stack_bwd_kept(storage_to_f64(dh), p64, caches)
    ref = {"h_out": h_out, "dh_in": dh_in, "grads": grads, "dcond": dcond}
    # the bound of the bf16 blocks for both storage types: a value next to a rounding border may take the other code
    errs = {n: gh.rel_err(a, b) for n, a, b in gh.pairs(got, ref, w.kind)}
    bad = {n: e for n, e in errs.items() if not e <= gh.tol_for("bf16")}
    assert not bad, bad
    # against the gradients of the unrounded activations: a code is off by at most half a step, a step at most 2/127
    # of its block's largest value, so under 1 % of the block's deviation in the mean (a uniform error over a step of
    # 0.034 of it); five kept tensors per block add up to about twice that, blocks add in squares
    for n, a, b in gh.pairs(got, dict(plain_f64(plain)), w.kind):
        if n != "h_out" and np.linalg.norm(b) > 0:
            assert np.linalg.norm(a - b) <= 0.05 * np.linalg.norm(b), n


def plain_f64(r):
    yield "h_out", storage_to_f64(r["h_out"])
    yield "dh_in", storage_to_f64(r["dh_in"])
    yield "grads", r["grads"]
    yield "dcond", r["dcond"]


def test_same_bits_whatever_the_scratch_held():
    w, nb = CASES["three_blocks"]
    h, params, cond, dh = gh.host_inputs(w, nb)
    a, _ = _run(w, w.L, h, params, cond, dh, True, scratch_fill=0xFF)
    b, _ = _run(w, w.L, h, params, cond, dh, True, scratch_fill=0x00)
    assert np.array_equal(a["dh_in"], b["dh_in"])
    for x, y in zip(a["grads"], b["grads"]):
        for k in x:
            assert np.array_equal(x[k], y[k]), k


@pytest.mark.parametrize("w", [inputs.small("save8_r", Hg=10, Wg=21), inputs.WORKLOADS["b5625"].with_(n_blocks=3)],
                         ids=["small", "b5625"])
def test_routed_calls_and_graph_replays(w):
    """sr_routed_blocks_fwd / _bwd with 8-bit saved activations equal gather + sparse calls + scatter, eagerly and
    in a replayed graph, and a second backward from the same saved activations gives the same bits."""
    import torch
    nb, K = w.n_blocks, w.K
    print(f"[save8 routed {w.name}] B={w.B} L={w.L} K={K}", flush=True)
    params = inputs.params_to_storage(inputs.block_params(w, nb, randomise_affine=True), w.dtype)
    cfg = device.config_for(w, n_blocks=nb)
    cfg.kind |= abi.SR_BLOCK_SAVE8
    dp, gr = device.DeviceParams(params, w.kind), device.DeviceGrads(w, nb, skip_unused=True)
    x0 = device.to_device(inputs.to_storage(inputs.token_field(w), w.dtype))
    g0 = device.to_device(inputs.to_storage(inputs.upstream_grad(w), w.dtype))
    idx = torch.empty((w.B, K), dtype=torch.int32, device="cuda")
    saved, scratch = device.workspace(cfg, K)
    abi.sr_select_indices(cfg, K, abi.SR_SEL_RANDOM, 9, 4, None, None, idx)
    x, g = x0.clone(), g0.clone()
    h0 = torch.empty((w.B, K, w.D), dtype=x.dtype, device="cuda")
    h, gh_, dh = torch.empty_like(h0), torch.empty_like(h0), torch.empty_like(h0)
    abi.sr_gather(cfg, K, x, idx, h0)
    abi.sr_sparse_blocks_fwd(cfg, K, dp.array, None, h0, h, saved)
    abi.sr_scatter_delta(cfg, K, x, h, h0, idx)
    abi.sr_gather(cfg, K, g, idx, gh_)
    abi.sr_sparse_blocks_bwd(cfg, K, dp.array, None, saved, gh_, dh, gr.array, None, scratch)
    abi.sr_scatter_delta(cfg, K, g, dh, None, idx)
    torch.cuda.synchronize()
    want = [x.clone(), g.clone()] + [v.clone() for t in gr.tensors for k, v in t.items() if not k.endswith("ada")]

    def step():
        abi.sr_routed_blocks_fwd(cfg, K, idx, dp.array, None, x, saved)
        abi.sr_routed_blocks_bwd(cfg, K, idx, dp.array, None, saved, g, gr.array, None, scratch)

    def check(tag):
        torch.cuda.synchronize()
        now = [x, g] + [v for t in gr.tensors for k, v in t.items() if not k.endswith("ada")]
        for i, (a, b) in enumerate(zip(now, want)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (tag, i)

    x.copy_(x0); g.copy_(g0); saved.fill_(0xEE)
    step()
    check("eager")
    g.copy_(g0)
    abi.sr_routed_blocks_bwd(cfg, K, idx, dp.array, None, saved, g, gr.array, None, scratch)
    check("second backward")
    graph = torch.cuda.CUDAGraph()
    x.copy_(x0); g.copy_(g0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        x.copy_(x0); g.copy_(g0); saved.fill_(0x11)
        torch.cuda.synchronize()
        graph.replay()
        check(("replay", rep))
        step()   # eager work between replays
        torch.cuda.synchronize()


@pytest.mark.parametrize("checkpoint", [False, True])
def test_trunk_with_8_bit_saved_activations(checkpoint):
    import torch
    w, split = inputs.small("save8_t", Hg=10, Wg=21), (1, 3, 1)
    params = inputs.params_to_storage(inputs.block_params(w, sum(split), randomise_affine=True), w.dtype)
    x0 = device.to_device(inputs.to_storage(inputs.token_field(w), w.dtype))
    g3 = device.to_device(inputs.to_storage(inputs.upstream_grad(w), w.dtype))
    runs = []
    for save8 in (False, True):
        tr = Trunk(w, split, params, seed=5, save8=save8, checkpoint=checkpoint)
        x3 = tr.forward(x0, 2).clone()
        g0 = tr.backward(g3).clone()
        torch.cuda.synchronize()
        runs.append((x3, g0, tr.block_grads(), sum({t.data_ptr(): t.numel() for t in tr.saved}.values())))
    (x3a, g0a, gra, _), (x3b, g0b, grb, _) = runs
    assert torch.equal(x3a, x3b)
    assert float((g0a.double() - g0b.double()).norm() / g0a.double().norm()) <= 0.05
    for i, (a, b) in enumerate(zip(gra, grb)):
        for k in a:
            if not k.endswith("ada"):
                assert float((a[k] - b[k]).norm()) <= 0.05 * float(a[k].norm()) + 1e-30, (i, k)


def test_non_finite_tokens_leave_other_samples_alone():
    w, nb = CASES["preln_bf16"]
    h, params, cond, dh = gh.host_inputs(w, nb)
    clean, _ = _run(w, w.L, h, params, cond, dh, True)
    h2 = h.copy()
    h2[0, 3, 7] = 0x7FC0   # NaN
    got, _ = _run(w, w.L, h2, params, cond, dh, True)
    assert np.array_equal(got["h_out"][1], clean["h_out"][1]) and np.array_equal(got["dh_in"][1], clean["dh_in"][1])
    assert not np.isfinite(storage_to_f64(got["dh_in"][0])).all()
