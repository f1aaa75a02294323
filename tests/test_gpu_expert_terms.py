"""Which terms a token's sum over its experts has, whichever kernels run: one
token by token, some tens over tiles of 64 rows, hundreds over larger ones."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from gpu_util import device, note

pytestmark = pytest.mark.gpu

COUNTS = [1, 2, 20, 200]


def _layer(seed, experts=4, hidden=256, inner=192):
    import torch
    g = torch.Generator().manual_seed(seed)

    def draw(*shape):
        return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device())

    return sp.Experts.from_dense(draw(experts, inner, hidden), draw(experts, inner, hidden),
                                 draw(experts, hidden, inner))


def _input(n, dtype, seed, experts=4, hidden=256, k=2):
    import torch
    from fp8_util import torch_dtype
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, hidden), generator=g).to(torch_dtype(dtype)).to(device())
    best = torch.randn((n, experts), generator=g).topk(k)
    return x, best.indices.int().to(device()), torch.softmax(best.values, 1).to(device())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", COUNTS)
def test_a_weight_of_zero_is_a_term(n, dtype):
    """0 * NaN is NaN; 0 times a finite row adds nothing."""
    import torch
    note("experts %s n %d, weights of zero" % (dtype, n))
    layer = _layer(1)
    x, ids, weights = _input(n, dtype, 2)
    weights[:, 1] = 0
    y = layer.run(x, ids, weights)
    ids[:, 1] = -1
    assert torch.equal(y, layer.run(x, ids, weights))
    x, ids, weights = _input(n, dtype, 2)
    x[n - 1, 7] = float("nan")
    weights[n - 1] = 0
    y = layer.run(x, ids, weights)
    assert y[n - 1].isnan().all() and y[:n - 1].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", COUNTS)
def test_an_id_of_no_expert_is_none(n, dtype):
    """Neither its weight nor any expert's parameters reach the sum."""
    note("experts %s n %d, ids of no expert" % (dtype, n))
    layer = _layer(3)
    layer.w13_scale[0] = float("nan")
    layer.w2_scale[0] = float("nan")
    x, ids, weights = _input(n, dtype, 4)
    ids[ids == 0] = 3
    clean = layer.run(x, ids, weights)
    assert clean.isfinite().all()
    ids[n - 1] = -1
    weights[n - 1] = float("nan")
    y = layer.run(x, ids, weights)
    assert (y[n - 1] == 0).all() and np.array_equal(y[:n - 1].float().cpu().numpy(), clean[:n - 1].float().cpu().numpy())
