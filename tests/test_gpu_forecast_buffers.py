"""Forecasts next to training on one trunk: a forecast, eager or replayed, leaves what the backward of a forward
reads alone, and new weights reach it."""
import pytest

from paper_2607_02829_amd import device, inputs
from paper_2607_02829_amd.trunk import Trunk

pytestmark = pytest.mark.gpu

W, SPLIT = inputs.small("b8_g", Hg=10, Wg=21), (1, 2, 1)


def _setup(checkpoint=False, save8=False):
    params = inputs.params_to_storage(inputs.block_params(W, sum(SPLIT), randomise_affine=True), W.dtype)
    x0, g3 = (device.to_device(inputs.to_storage(f(W), W.dtype)) for f in (inputs.token_field, inputs.upstream_grad))
    return Trunk(W, SPLIT, params, seed=7, checkpoint=checkpoint, save8=save8), x0, g3


def _grads(tr, g0):
    import torch
    torch.cuda.synchronize()
    return [g0.clone()] + [t.clone() for g in tr.block_grads() for k, t in sorted(g.items()) if not k.endswith("ada")]


def _same(a, b):
    import torch
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b, strict=True))


def _capture(run):
    import torch
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    return graph


@pytest.mark.parametrize("checkpoint,save8", [(False, False), (True, False), (False, True), (True, True)])
def test_a_replayed_forecast_leaves_the_backward_alone(checkpoint, save8):
    import torch
    tr, x0, g3 = _setup(checkpoint, save8)
    x3 = tr.forward(x0, 3).clone()
    idx = tr.idx.clone()
    want = _grads(tr, tr.backward(g3))
    tr.quantize()
    graph = _capture(lambda: tr.forecast(x0, 9))   # other indices
    graph.replay()
    torch.cuda.synchronize()
    y = tr.x3.clone()
    for rep in range(3):
        assert torch.equal(tr.forward(x0, 3), x3) and torch.equal(tr.idx, idx)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tr.x3, y), rep
        assert _same(_grads(tr, tr.backward(g3)), want), rep


def test_capturing_a_forecast_leaves_the_backward_allowed():
    import torch
    tr, x0, g3 = _setup()
    tr.quantize()
    tr.forecast(x0, 9)
    tr.forward(x0, 3)
    want = _grads(tr, tr.backward(g3))
    tr.forward(x0, 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):   # nothing runs yet
        tr.forecast(x0, 9)
    assert _same(_grads(tr, tr.backward(g3)), want)


def test_backward_of_a_replayed_forward_after_a_forecast():
    import torch
    tr, x0, g3 = _setup()
    tr.quantize()
    tr.forward(x0, 3)
    want = _grads(tr, tr.backward(g3))
    graph = _capture(lambda: tr.forward(x0, 3))
    for rep in range(3):
        tr.forecast(x0, 9)
        graph.replay()
        assert _same(_grads(tr, tr.backward(g3)), want), rep


def test_new_weights_change_a_captured_forecast():
    import torch
    tr, x0, _ = _setup()
    tr.quantize()
    graph = _capture(lambda: tr.forecast(x0, 3))
    graph.replay()
    torch.cuda.synchronize()
    before = tr.x3.clone()
    for p in tr.params:
        for t in p.tensors:
            t["w_fc2"].mul_(2.0)
    tr.quantize()
    # a trunk that was built from and quantised with the new weights
    params = inputs.params_to_storage(inputs.block_params(W, sum(SPLIT), randomise_affine=True), W.dtype)
    fresh = Trunk(W, SPLIT, params, seed=7)
    for p in fresh.params:
        for t in p.tensors:
            t["w_fc2"].mul_(2.0)
    fresh.quantize()
    want = fresh.forecast(x0, 3).clone()
    torch.cuda.synchronize()
    assert not torch.equal(want, before)
    for rep in range(3):
        tr.x3.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tr.x3.view(torch.int16), want.view(torch.int16)), rep
        assert torch.equal(tr.forecast(x0, 3).view(torch.int16), want.view(torch.int16)), rep
