"""Experts are off by their result's rounding and little else, in every type and over
tiles of 64 and of 128 rows, also where a few channels of a row are much louder
than the rest (the 8-bit instruction's cut grows with them, 32-bit sums do not)."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from expert_bounds import BESIDES, norm_error, reference
from fp8_util import torch_dtype
from gpu_util import device, note

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,experts,k,hidden,inner", [(2000, 512, 8, 200, 264), (1030, 20, 8, 256, 520), (9000, 5, 4, 140, 128)])
def test_little_beside_the_rounding(dtype, n, experts, k, hidden, inner):
    """The error's norm against the rounding's, and what else there may be, as independent of each other."""
    import torch
    note("experts %s n %d of %d, %d x %d, loud channels" % (dtype, n, experts, hidden, inner))
    g = torch.Generator().manual_seed(n)

    def draw(*shape):
        return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device())

    layer = sp.Experts.from_dense(draw(experts, inner, hidden), draw(experts, inner, hidden),
                                  draw(experts, hidden, inner))
    x = torch.randn((n, hidden), generator=g)
    x[:, torch.randint(0, hidden, (2,), generator=g)] *= 10
    x = x.to(torch_dtype(dtype)).to(device())
    best = torch.randn((n, experts), generator=g).topk(k)
    ids, weights = best.indices.int().to(device()), torch.softmax(best.values, 1).to(device())
    y = layer.run(x, ids, weights)
    ref = reference(x.float().cpu().numpy(), ids.cpu().numpy(), weights.cpu().numpy(), layer)
    rounding = norm_error(torch.from_numpy(ref).to(torch_dtype(dtype)), ref)
    # one code of a value of four times the usual size besides
    others = BESIDES[dtype] + 4 * 2.0 ** -3 / (n * k * inner) ** 0.5
    got = norm_error(y, ref)
    assert got <= 1.05 * (rounding ** 2 + others ** 2) ** 0.5, "%.3g, the rounding alone %.3g" % (got, rounding)
    assert np.isfinite(got)
