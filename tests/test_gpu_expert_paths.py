"""Experts at the sizes that choose each way through the kernels: long rows and
many choices of a single token, more experts than a wavefront has lanes, sorts of
thousands of pairs, whole-line stores of the largest tiles; and that f32 and f16
keep their exact products."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from expert_bounds import NORM, bound, norm_error, reference
from fp8_util import torch_dtype
from gpu_util import device, note

pytestmark = pytest.mark.gpu

DTYPES = ["f32", "f16", "bf16"]


def _layer(experts, hidden, inner, seed):
    import torch
    g = torch.Generator().manual_seed(seed)

    def draw(*shape):
        return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device())

    return sp.Experts.from_dense(draw(experts, inner, hidden), draw(experts, inner, hidden),
                                 draw(experts, hidden, inner))


def _input(n, experts, k, hidden, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, hidden), generator=g).to(torch_dtype(dtype)).to(device())
    best = (torch.randn((n, experts), generator=g) + torch.randn(experts, generator=g)).topk(k)
    return x, best.indices.int().to(device()), torch.softmax(best.values, 1).to(device())


def _numpy(*tensors):
    return [t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy() for t in tensors]


def _each(y, x, ids, weights, layer, dtype):
    """Every element within its bound."""
    ref, tol = bound(*_numpy(x, ids, weights), layer, dtype)
    err = np.abs(y.double().cpu().numpy() - ref)
    assert y.dtype == torch_dtype(dtype) and y.shape == ref.shape
    assert (err <= tol).all(), "worst error / tolerance %.3g" % float((err / tol).max())


def _together(y, x, ids, weights, layer, dtype):
    """All of them within what well spread inputs allow, and one code of a value of four times the usual size."""
    pairs = int((ids >= 0).sum())
    got = norm_error(y, reference(*_numpy(x, ids, weights), layer))
    assert got <= NORM[dtype] + 4 * 2.0 ** -3 / (pairs * layer.inner) ** 0.5, "relative error %.3g" % got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,experts,k,hidden,inner", [
    (1, 8, 2, 2049, 128), (1, 8, 1, 4100, 300), (2, 16, 3, 6150, 200),    # rows of more than 2048 channels
    (1, 8, 6, 256, 2048), (2, 24, 9, 130, 1025), (1, 4, 2, 200, 8200),    # more than 8 thousands of inner channels
    (1, 16, 7, 2300, 1500), (8, 64, 4, 2100, 130),
])
def test_long_rows_of_single_tokens(dtype, n, experts, k, hidden, inner):
    note("experts %s n %d of %d, %d x %d" % (dtype, n, experts, hidden, inner))
    layer = _layer(experts, hidden, inner, hidden + inner)
    x, ids, weights = _input(n, experts, k, hidden, dtype, n + k)
    _each(layer.run(x, ids, weights), x, ids, weights, layer, dtype)
    ids[0, k - 1] = -1
    _each(layer.run(x, ids, weights), x, ids, weights, layer, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,experts,k,hidden,inner", [(20, 65, 4, 128, 256), (100, 129, 6, 200, 130), (9, 300, 8, 128, 128),
                                                      (700, 1024, 4, 130, 100)])
def test_more_experts_than_lanes(dtype, n, experts, k, hidden, inner):
    note("experts %s n %d of %d, %d x %d" % (dtype, n, experts, hidden, inner))
    layer = _layer(experts, hidden, inner, experts)
    x, ids, weights = _input(n, experts, k, hidden, dtype, n)
    ids[1, 0] = experts - 1
    ids[2, 0] = 64
    ids[3, 1] = experts
    _each(layer.run(x, ids, weights), x, ids, weights, layer, dtype)


# from 4096 pairs on rows are prepared by 1024 threads; past 32768 ids are read twice; four blocks
# of a row at once from 1024 groups and blocks on
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,experts,k,hidden,inner", [(9000, 5, 4, 128, 128), (8193, 130, 4, 140, 200), (1100, 4, 4, 7900, 128),
                                                      (600, 6, 2, 3500, 130), (1030, 20, 8, 256, 520)])
def test_thousands_of_pairs(dtype, n, experts, k, hidden, inner):
    import torch
    note("experts %s n %d of %d, %d x %d" % (dtype, n, experts, hidden, inner))
    layer = _layer(experts, hidden, inner, hidden)
    x, ids, weights = _input(n, experts, k, hidden, dtype, n)
    ids[torch.randperm(n, generator=torch.Generator().manual_seed(1))[:n // 50].to(ids.device), 0] = -1
    y = layer.run(x, ids, weights)
    _together(y, x, ids, weights, layer, dtype)
    some = torch.arange(0, n, 37, device=ids.device)
    _each(y[some], x[some], ids[some], weights[some], layer, dtype)
    assert torch.equal(y, layer.run(x, ids, weights))


# whole lines of results: tiles of 256 rows (200 rows an expert, 11 column tiles), 128 and 64
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,experts,k,hidden,inner", [(800, 8, 2, 2816, 200), (560, 8, 2, 2304, 136), (800, 8, 2, 2820, 1408),
                                                      (100, 4, 2, 512, 640)])
def test_whole_lines(dtype, n, experts, k, hidden, inner):
    note("experts %s n %d of %d, %d x %d" % (dtype, n, experts, hidden, inner))
    layer = _layer(experts, hidden, inner, inner)
    x, ids, weights = _input(n, experts, k, hidden, dtype, n)
    y = layer.run(x, ids, weights)
    _each(y, x, ids, weights, layer, dtype)
    _together(y, x, ids, weights, layer, dtype)


# Inner rows that are codes as they are: a gate of 448 * 448, whose silu is itself, times 448 * x for a
# channel x of the row that is one code; so only the second products are off.  Their sums of 640 terms in 32
# bits are about sqrt(640) * 2^-24 = 1.5e-6 of their size off at most, sums on the 8-bit instruction 4e-5.
@pytest.mark.parametrize("n", [1, 20, 200, 800])
def test_second_products_in_32_bits(n):
    import torch
    note("experts f32 n %d, inner rows that are codes" % n)
    size, g = 640, torch.Generator().manual_seed(n)
    x = (torch.randn((n, size), generator=g) * 60).clamp(-440, 440).to(torch.float8_e4m3fn).float()
    x[:, ::128] = 448.0
    w1, w3 = torch.zeros((1, size, size)), torch.zeros((1, size, size))
    w1[0, :, 0] = 448.0
    w3[0, torch.arange(size), torch.arange(size)] = 448.0
    w2 = torch.randn((1, size, size), generator=g) * 1e-11
    x, w1, w3, w2 = (t.to(device()) for t in (x, w1, w3, w2))
    layer = sp.Experts.from_dense(w1, w3, w2)
    ids = torch.zeros((n, 1), dtype=torch.int32, device=device())
    weights = torch.ones((n, 1), device=device())
    y = layer.run(x, ids, weights)
    inner = x.double().cpu().numpy() * 448.0 ** 3
    values = (layer.w2[0].double().cpu() * layer.w2_scale[0].double().cpu().repeat_interleave(128, 0)
              .repeat_interleave(128, 1)).numpy()
    assert norm_error(y, inner @ values.T) <= 4e-6
