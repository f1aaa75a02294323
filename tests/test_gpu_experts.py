"""Routers and experts (spconv_route, spconv_experts_fp8) against 64-bit references.

A router's ids are held to equality (its values are 64-bit on both sides), its
weights to one rounding to 32 bits.  Experts are held to fp8_util.experts_ref's
bound, which follows 32-bit sums through the gate and the rounding of the inner
rows to codes.
"""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import ROUND, SMALLEST, experts_ref, route_ref, torch_dtype
from gpu_util import device, note

pytestmark = pytest.mark.gpu


def _check_route(logits, k, **kw):
    bias = kw.get("bias")
    ids, weights = sp.route(logits, k, **kw)
    kw["bias"] = None if bias is None else bias.cpu().numpy()
    ref_ids, ref_w = route_ref(logits.float().cpu().numpy(), k, **kw)
    assert np.array_equal(ids.cpu().numpy(), ref_ids)
    assert np.allclose(weights.cpu().numpy(), ref_w, rtol=2.0 ** -23, atol=1e-38)


def _logits(n, experts, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, experts), generator=g) * 1.5).to(torch_dtype(dtype)).to(device())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n,experts,k,groups,kept,top", [
    (1, 1, 1, 1, 1, 1), (1, 64, 6, 1, 1, 1), (5, 8, 8, 1, 1, 1), (67, 60, 4, 1, 1, 1), (3, 65, 5, 1, 1, 1),
    (33, 128, 8, 8, 3, 2), (9, 160, 6, 8, 3, 1), (40, 256, 8, 8, 4, 2), (6, 257, 8, 1, 1, 1), (7, 500, 10, 10, 5, 2),
    (4, 1000, 64, 1, 1, 1), (3, 1024, 16, 64, 2, 2), (5, 12, 3, 12, 5, 1), (11, 21, 2, 3, 1, 2),
])
def test_route_matches_64_bits(dtype, score, n, experts, k, groups, kept, top):
    note("route %s %s n %d experts %d k %d groups %d" % (dtype, score, n, experts, k, groups))
    import torch
    logits = _logits(n, experts, dtype, n + experts)
    bias = (torch.randn(experts, generator=torch.Generator().manual_seed(1)) * 0.1).to(device())
    for b in (None, bias):
        for renorm, factor in ((True, 1.0), (False, 2.5)):
            _check_route(logits, k, score=score, bias=b, groups=groups, groups_kept=kept, group_top=top,
                         renorm=renorm, factor=factor)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_equal_values_go_to_the_lowest_index(score):
    import torch
    logits = torch.zeros((4, 96), device=device())
    logits[1, 40:44] = 1.0
    logits[2, ::5] = -2.0
    logits[3] = torch.finfo(torch.float32).min
    _check_route(logits, 7, score=score)
    _check_route(logits, 7, score=score, groups=8, groups_kept=3, group_top=2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,kept", [(1, 1), (4, 2)])
def test_route_experts_that_are_off(score, groups, kept):
    import torch
    logits = _logits(7, 72, "f32", 5)
    logits[0] = -float("inf")                  # none left
    logits[1, 3:] = -float("inf")              # fewer than k
    logits[2, 10:30] = float("nan")
    logits[3, 5] = float("inf")
    logits[4, :36] = -float("inf")             # whole groups
    logits[5, 7] = torch.finfo(torch.float32).min
    bias = torch.zeros(72, device=device())
    bias[60] = -float("inf")
    bias[61] = -5.0
    _check_route(logits, 6, score=score, groups=groups, groups_kept=kept, group_top=2, bias=bias)
    ids, weights = sp.route(logits, 6, score=score, groups=groups, groups_kept=kept)
    assert (ids[0] == -1).all() and (weights[0] == 0).all()


def test_route_strided_logits_and_many_tokens():
    wide = _logits(9000, 100, "bf16", 3)
    _check_route(wide[:, 3:67], 6, score="sigmoid")
    _check_route(wide[::7, :64], 2)


def _experts(experts, hidden, inner, seed):
    import torch
    g = torch.Generator().manual_seed(seed)

    def draw(*shape):
        return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device())

    return sp.Experts.from_dense(draw(experts, inner, hidden), draw(experts, inner, hidden),
                                 draw(experts, hidden, inner))


def _rows(n, cols, dtype, seed, extra=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, cols + extra), generator=g).to(torch_dtype(dtype)).to(device())[:, :cols]


def _chosen(n, k, experts, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    skew = torch.randn(experts, generator=g)
    best = (torch.randn((n, experts), generator=g) + skew).topk(k)
    return best.indices.int().to(device()), torch.softmax(best.values, 1).to(device())


def _check_experts(y, x, ids, weights, layer, dtype):
    ref, tol = experts_ref(x.float().cpu().numpy(), ids.cpu().numpy(), weights.cpu().numpy(), layer,
                           cut=dtype != "f32")
    tol = tol + np.abs(ref) * ROUND[dtype] + SMALLEST[dtype]
    err = np.abs(y.double().cpu().numpy() - ref)
    assert y.shape == ref.shape and y.dtype == torch_dtype(dtype)
    assert (err <= tol).all(), "worst error / tolerance %.3g" % float((err / tol).max())
    # the bound of one element allows a code of every inner channel to differ; together they do not
    norm = float(np.linalg.norm(ref))
    if norm:
        assert np.linalg.norm(err) <= norm * (2 * ROUND[dtype] + 5e-3)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,experts,k,hidden,inner,extra", [
    (1, 1, 1, 1, 1, 0), (1, 8, 2, 128, 128, 0), (1, 16, 6, 300, 200, 0), (3, 4, 4, 257, 130, 1), (4, 64, 8, 512, 96, 8),
    (5, 8, 2, 256, 128, 0), (16, 3, 2, 130, 257, 2), (50, 32, 4, 640, 200, 0), (30, 2, 1, 128, 384, 0),
    (40, 2, 2, 384, 256, 0), (130, 4, 2, 200, 130, 3), (300, 3, 2, 513, 129, 0), (260, 2, 2, 256, 640, 0),
])
def test_experts_match_64_bits(dtype, n, experts, k, hidden, inner, extra):
    note("experts %s n %d experts %d k %d hidden %d inner %d" % (dtype, n, experts, k, hidden, inner))
    layer = _experts(experts, hidden, inner, n + hidden)
    x = _rows(n, hidden, dtype, inner, extra)
    ids, weights = _chosen(n, k, experts, n)
    _check_experts(layer.run(x, ids, weights), x, ids, weights, layer, dtype)


# few tokens of small experts, on both sides of where they are taken one by one
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,experts,k,hidden,inner", [(3, 16, 4, 300, 200), (8, 32, 4, 1000, 130), (8, 9, 1, 257, 1030),
                                                      (9, 32, 2, 300, 200), (8, 31, 4, 300, 200), (5, 64, 6, 1300, 900)])
def test_experts_few_tokens(dtype, n, experts, k, hidden, inner):
    note("experts %s n %d experts %d k %d hidden %d inner %d" % (dtype, n, experts, k, hidden, inner))
    layer = _experts(experts, hidden, inner, n + hidden)
    x = _rows(n, hidden, dtype, inner, 0)
    ids, weights = _chosen(n, k, experts, n)
    ids[n - 1, 0] = -1
    ids[0, k - 1] = ids[1, k - 1]
    _check_experts(layer.run(x, ids, weights), x, ids, weights, layer, dtype)


# enough tiles for those of 256 and of 128 rows, with parts of them empty
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,experts,k,hidden,inner", [(800, 8, 2, 300, 1410), (801, 8, 2, 2820, 200),
                                                      (800, 8, 2, 2819, 130), (560, 8, 2, 300, 1157),
                                                      (560, 8, 2, 2304, 200)])
def test_experts_large_tiles(dtype, n, experts, k, hidden, inner):
    note("experts %s n %d experts %d k %d hidden %d inner %d" % (dtype, n, experts, k, hidden, inner))
    layer = _experts(experts, hidden, inner, n + hidden)
    x = _rows(n, hidden, dtype, inner, 0)
    ids, weights = _chosen(n, k, experts, n)
    _check_experts(layer.run(x, ids, weights), x, ids, weights, layer, dtype)


@pytest.mark.parametrize("n,experts", [(2, 8), (40, 8), (200, 2)])
def test_experts_ids_that_are_none(n, experts):
    import torch
    layer = _experts(experts, 256, 192, 2)
    x = _rows(n, 256, "f32", 3)
    ids, weights = _chosen(n, 2, experts, 4)
    ids[0] = -1
    ids[1, 0] = experts
    ids[n - 1, 1] = 2 ** 31 - 1
    y = layer.run(x, ids, weights)
    _check_experts(y, x, ids, weights, layer, "f32")
    assert (y[0] == 0).all()
    ids[:] = -1
    assert (layer.run(x, ids, weights) == 0).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("n", [3, 30, 200])
def test_experts_all_tokens_to_one_expert(n):
    import torch
    layer = _experts(4, 256, 256, 2)
    x = _rows(n, 256, "f16", 3)
    ids = torch.full((n, 1), 2, dtype=torch.int32, device=device())
    weights = torch.ones((n, 1), device=device())
    _check_experts(layer.run(x, ids, weights), x, ids, weights, layer, "f16")


@pytest.mark.parametrize("n", [4, 60, 300])
def test_experts_a_row_that_is_not_finite_changes_no_other(n):
    import torch
    layer = _experts(4, 256, 256, 2)
    x = _rows(n, 256, "bf16", 3)
    ids, weights = _chosen(n, 2, 4, 4)
    clean = layer.run(x, ids, weights)
    x[1, 7] = float("inf")
    x[2, 255] = float("nan")
    y = layer.run(x, ids, weights)
    keep = torch.ones(n, dtype=torch.bool, device=x.device)
    keep[1] = keep[2] = False
    assert torch.equal(y[keep], clean[keep])
    assert y[1].isnan().all() and y[2].isnan().all()


def test_experts_large_gates():
    """exp(-gate) past the range of 32 bits on both sides."""
    import torch
    layer = _experts(2, 128, 128, 2)
    x = _rows(8, 128, "f32", 3) * torch.logspace(0, 12, 8, device=device())[:, None]
    ids, weights = _chosen(8, 1, 2, 4)
    y = layer.run(x, ids, weights)
    assert y.isfinite().all()
    _check_experts(y, x, ids, weights, layer, "f32")


@pytest.mark.parametrize("n", [1, 20, 200])
def test_experts_on_another_stream_and_in_a_graph(n):
    import torch
    layer = _experts(4, 256, 256, 2)
    x = _rows(n, 256, "bf16", 3)
    ids, weights = _chosen(n, 2, 4, 4)
    ref = layer.run(x, ids, weights).clone()
    y = torch.empty_like(ref)
    space = torch.empty(layer.workspace_bytes(n, 2), dtype=torch.uint8, device=device())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer.run(x, ids, weights, y, space, side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(x, ids, weights, y, space)
    for r in range(3):
        x.copy_(_rows(n, 256, "bf16", 20 + r))
        i, w = _chosen(n, 2, 4, 30 + r)
        ids.copy_(i)
        weights.copy_(w)
        space.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, layer.run(x, ids, weights)), "replay %d" % r


def test_experts_empty_run():
    import torch
    layer = _experts(4, 256, 256, 2)
    y = layer.run(torch.empty((0, 256), device=device()), torch.empty((0, 2), dtype=torch.int32, device=device()),
                  torch.empty((0, 2), device=device()))
    assert y.shape == (0, 256)
