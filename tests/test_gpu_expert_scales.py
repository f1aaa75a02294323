"""Experts whose weights' scales have either sign: a value is its code times its
block's scale, whatever the scale."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from expert_bounds import NORM, bound, norm_error
from fp8_util import torch_dtype
from gpu_util import device, note

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,experts,hidden,inner", [(1, 4, 300, 640), (30, 4, 256, 384), (200, 2, 256, 640),
                                                    (260, 1, 384, 256)])
def test_scales_of_either_sign(dtype, n, experts, hidden, inner):
    import torch
    note("experts %s n %d of %d, %d x %d, signed scales" % (dtype, n, experts, hidden, inner))
    g = torch.Generator().manual_seed(n + hidden)

    def draw(*shape):
        return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device())

    layer = sp.Experts.from_dense(draw(experts, inner, hidden), draw(experts, inner, hidden),
                                  draw(experts, hidden, inner))
    for scale in (layer.w13_scale, layer.w2_scale):
        sign = torch.randint(0, 2, scale.shape, generator=g).to(scale) * 2 - 1
        scale.mul_(sign)
    x = torch.randn((n, hidden), generator=g).to(torch_dtype(dtype)).to(device())
    k = min(2, experts)
    best = torch.randn((n, experts), generator=g).topk(k)
    ids, weights = best.indices.int().to(device()), torch.softmax(best.values, 1).to(device())
    y = layer.run(x, ids, weights)
    ref, tol = bound(x.float().cpu().numpy(), ids.cpu().numpy(), weights.cpu().numpy(), layer, dtype)
    err = np.abs(y.double().cpu().numpy() - ref)
    assert (err <= tol).all(), "worst error / tolerance %.3g" % float((err / tol).max())
    if n > 1:  # a row alone is too few to average over
        assert norm_error(y, ref) <= NORM[dtype]
