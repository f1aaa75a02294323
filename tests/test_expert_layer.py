"""The operators of an expert layer together (ExpertLayer), on the GPU."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import ROUND, block_values, code_values, experts_ref, linear_tol, quantize_ref, route_ref, row_values, torch_dtype
from gpu_util import device, note

pytestmark = pytest.mark.gpu


def _layer(dtype, batch, experts, k, hidden, inner, cout, seed, **choice):
    import torch
    g = torch.Generator().manual_seed(seed)

    def draw(*shape):
        return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device())

    nets = sp.Experts.from_dense(draw(experts, inner, hidden), draw(experts, inner, hidden),
                                 draw(experts, hidden, inner))
    head = sp.Fp8Linear.from_dense(draw(cout, hidden), draw(cout), "relu6")
    bias = (torch.randn(experts, generator=g) * 0.05).to(device())
    return sp.ExpertLayer(draw(experts, hidden) * 8, nets, k, batch, torch_dtype(dtype), head, bias=bias, **choice)


def _input(batch, hidden, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn((batch, hidden), generator=g).to(torch_dtype(dtype)).to(device())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("batch", [1, 13, 200])
def test_steps_follow_each_other(dtype, batch):
    """Each step's output against the reference on what the step before left."""
    note("expert layer %s batch %d" % (dtype, batch))
    choice = dict(score="sigmoid", groups=4, groups_kept=2, group_top=2, factor=2.5)
    layer = _layer(dtype, batch, 16, 3, 320, 200, 150, 1, **choice)
    x = _input(batch, 320, dtype, 2)
    out = layer.forward(x)
    xf = x.float().cpu().numpy()
    router = layer.router.cpu().double().numpy()
    logits = layer.logits.cpu().numpy()
    ref = xf.astype(np.float64) @ router.T
    terms = np.abs(xf).astype(np.float64) @ np.abs(router).T
    assert (np.abs(logits - ref) <= terms * 340 * 2.0 ** -24).all()
    ids, weights = route_ref(logits, 3, bias=layer.choice["bias"].cpu().numpy(), **choice)
    assert np.array_equal(layer.ids.cpu().numpy(), ids)
    assert np.allclose(layer.weights.cpu().numpy(), weights, rtol=2.0 ** -23, atol=0)
    y, tol = experts_ref(xf, ids, layer.weights.cpu().numpy(), layer.experts, cut=dtype != "f32")
    r = ROUND[dtype]
    got = layer.y.cpu().double().numpy()  # rounded once by the experts and once by the residual sum
    assert (np.abs(got - (y + xf)) <= tol + (np.abs(y) + np.abs(got)) * 1.01 * r + 1e-6).all()
    q, s = quantize_ref(layer.y.float().cpu().numpy(), 1)
    xv = row_values(q, s, 320)
    wv = block_values(code_values(layer.head.w), layer.head.w_scale.cpu().numpy(), 320)
    b = layer.head.bias.cpu().double().numpy()
    ref = np.clip(xv @ wv.T + b, 0, 6)
    tol = linear_tol(ref, np.abs(xv) @ np.abs(wv).T + np.abs(b), 320, dtype)
    assert (np.abs(out.cpu().double().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("batch", [1, 50])
def test_replays_equal_eager_runs(batch):
    import torch
    layer = _layer("bf16", batch, 8, 2, 256, 128, 100, 3)
    layer.capture()
    for r in range(3):
        x = _input(batch, 256, "bf16", 10 + r)
        layer.x.copy_(x)
        got = layer.replay().clone()
        torch.cuda.synchronize()
        assert torch.equal(got, layer.forward(x)), "replay %d" % r
