"""8-bit blocks and dense layers on them (spconv_quantize_fp8, spconv_linear_fp8)
against 64-bit references.

Codes and scales are held to equality: every step of their definition is one
correctly rounded 32-bit operation.  Products are held to the bound of
fp8_util.linear_tol.
"""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import (BLOCK, block_values, blocks, code_values, linear_ref, linear_tol, quantize_ref, row_values,
                      torch_dtype)
from gpu_util import device, note

pytestmark = pytest.mark.gpu


def _rows(rows, cols, dtype, seed, extra=0):
    """A [rows, cols] matrix whose row stride is `extra` elements longer."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols + extra), generator=g) * torch.exp(torch.randn((rows, 1), generator=g))
    return x.to(torch_dtype(dtype)).to(device())[:, :cols]


def _check_codes(q, scale, x, block_rows):
    ref_q, ref_s = quantize_ref(x.float().cpu().numpy(), block_rows)
    assert np.array_equal(scale.cpu().numpy(), ref_s, equal_nan=True)
    assert np.array_equal(code_values(q), ref_q, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,extra", [(1, 1, 0), (1, 128, 0), (3, 127, 0), (17, 129, 0), (128, 256, 0),
                                             (129, 640, 8), (5, 300, 3), (300, 1000, 0), (70, 8192, 0)])
def test_quantize_equals_the_definition(dtype, block_rows, rows, cols, extra):
    note("quantize %s %d x %d + %d, blocks of %d" % (dtype, rows, cols, extra, block_rows))
    x = _rows(rows, cols, dtype, rows + cols, extra)
    q, scale = sp.quantize_fp8(x, block_rows)
    assert q.shape == (rows, blocks(cols) * BLOCK)
    _check_codes(q, scale, x, block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_zeros_tiny_huge_and_not_finite(block_rows):
    import torch
    x = torch.zeros((140, 512))
    x[0, 0:128] = torch.linspace(-1e-38, 1e-38, 128)           # below the floor of a scale
    x[1, 128:256] = 2.0 ** -100
    x[2, 300] = 3.4e38
    x[131, 5] = float("inf")                                   # in the second row of blocks
    x[132, 130] = float("nan")
    x[133, 256:384] = torch.arange(128) * (448.0 / 448) / 8    # values between two codes
    x = x.to(device())
    q, scale = sp.quantize_fp8(x, block_rows)
    _check_codes(q, scale, x, block_rows)
    if block_rows == 1:
        assert scale[0, 131].isinf() and scale[1, 132].isnan()
        fine = torch.ones_like(scale, dtype=torch.bool)
        fine[0, 131] = fine[1, 132] = False
        assert scale[fine].isfinite().all()


def _layer(cout, cin, seed, bias):
    import torch
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn((cout, cin), generator=g) / cin ** 0.5).to(device())
    b = torch.randn(cout, generator=g).to(device()) if bias else None
    return w, b


def _check_linear(y, x, layer, bias, act, dtype, quantized=None):
    if quantized is None:
        q, s = quantize_ref(x.float().cpu().numpy(), 1)
    else:
        q, s = code_values(quantized[0]), quantized[1].cpu().numpy()
    xv = row_values(q, s, layer.cin)
    wv = block_values(code_values(layer.w), layer.w_scale.cpu().numpy(), layer.cin)
    ref, terms = linear_ref(xv, wv, None if bias is None else bias.cpu().numpy(), act)
    err = np.abs(y.double().cpu().numpy() - ref)
    tol = linear_tol(ref, terms, layer.cin, dtype)
    assert y.dtype == torch_dtype(dtype) and y.shape == ref.shape
    assert (err <= tol).all(), "worst error / tolerance %.3g" % float((err / tol).max())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout,act,bias,extra", [
    (1, 1, 1, "none", False, 0), (1, 128, 16, "relu", True, 0), (1, 1000, 1000, "none", True, 0),
    (2, 4096, 129, "relu6", True, 0), (15, 384, 200, "none", False, 3), (16, 130, 127, "none", True, 8),
    (17, 1280, 320, "relu", False, 0), (31, 257, 6, "none", True, 1), (33, 512, 512, "none", False, 0),
    (64, 2176, 96, "none", True, 0), (65, 256, 256, "relu6", True, 0), (130, 100, 130, "none", False, 4),
    (200, 1024, 1000, "none", True, 0), (257, 640, 385, "relu", True, 0),
])
def test_linear_matches_64_bits(dtype, n, cin, cout, act, bias, extra):
    note("linear %s n %d cin %d cout %d %s" % (dtype, n, cin, cout, act))
    w, b = _layer(cout, cin, n + cin, bias)
    layer = sp.Fp8Linear.from_dense(w, b, act)
    x = _rows(n, cin, dtype, cout, extra)
    _check_linear(layer.run(x), x, layer, b, act, dtype)


# every tile shape, and grids of several thousand tiles
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout", [(70, 1300, 70), (300, 640, 2100), (1030, 384, 1030), (2050, 256, 2050),
                                        (4099, 384, 3075), (12, 128, 70000), (70000, 128, 12), (500, 2200, 3900),
                                        (450, 260, 4100), (790, 1100, 4000)])
def test_linear_many_rows_or_channels(dtype, n, cin, cout):
    note("linear %s n %d cin %d cout %d" % (dtype, n, cin, cout))
    w, b = _layer(cout, cin, 3, True)
    layer = sp.Fp8Linear.from_dense(w, b)
    x = _rows(n, cin, dtype, 4)
    _check_linear(layer.run(x), x, layer, b, "none", dtype)


# few rows: quantised in the product or before it, one or two pieces of channels a workgroup
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout", [(1, 2100, 8211), (9, 2100, 8211), (17, 4500, 8211), (32, 640, 8200),
                                        (3, 8100, 70), (20, 4224, 300), (32, 900, 2050), (8, 2049, 8190),
                                        (2, 5000, 5150), (27, 4090, 4100), (5, 1030, 25000), (50, 300, 24700)])
def test_linear_few_rows(dtype, n, cin, cout):
    note("linear %s n %d cin %d cout %d" % (dtype, n, cin, cout))
    w, b = _layer(cout, cin, 5, True)
    layer = sp.Fp8Linear.from_dense(w, b)
    x = _rows(n, cin, dtype, 6, 1)
    _check_linear(layer.run(x), x, layer, b, "none", dtype)


# many input channels and few tiles: workgroups share a tile's input channels
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout,act", [(33, 2048, 1, "none"), (40, 8192, 130, "relu"), (100, 4100, 66, "none"),
                                            (65, 16400, 64, "relu6"), (300, 2300, 257, "none"), (129, 8070, 515, "none")])
def test_linear_many_input_channels(dtype, n, cin, cout, act):
    note("linear %s n %d cin %d cout %d" % (dtype, n, cin, cout))
    w, b = _layer(cout, cin, 7, True)
    layer = sp.Fp8Linear.from_dense(w, b, act)
    x = _rows(n, cin, dtype, 8)
    _check_linear(layer.run(x), x, layer, b, act, dtype)
    q = sp.quantize_fp8(x)
    _check_linear(layer.run(q[0], q[1], dtype=torch_dtype(dtype)), x, layer, b, act, dtype, q)


@pytest.mark.parametrize("n", [1, 16, 17, 40, 64, 65, 300])
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
def test_linear_of_quantised_rows(n, out):
    note("linear of codes n %d to %s" % (n, out))
    w, b = _layer(264, 700, n, True)
    layer = sp.Fp8Linear.from_dense(w, b, "relu")
    x = _rows(n, 700, "f32", 9)
    q = sp.quantize_fp8(x)
    y = layer.run(q[0], q[1], dtype=torch_dtype(out))
    _check_linear(y, x, layer, b, "relu", out, q)


@pytest.mark.parametrize("n", [4, 20, 100, 600])
def test_a_row_that_is_not_finite_changes_no_other(n):
    import torch
    w, b = _layer(300, 512, 5, True)
    layer = sp.Fp8Linear.from_dense(w, b)
    x = _rows(n, 512, "f32", 6)
    clean = layer.run(x)
    x[1, 200] = float("inf")
    x[3, 511] = float("nan")
    y = layer.run(x)
    keep = torch.ones(n, dtype=torch.bool, device=x.device)
    keep[1] = keep[3] = False
    assert torch.equal(y[keep], clean[keep])
    assert y[1].isnan().all() and y[3].isnan().all()


def test_activation_keeps_a_nan():
    w, b = _layer(32, 128, 5, False)
    layer = sp.Fp8Linear.from_dense(w, b, "relu6")
    x = _rows(2, 128, "f32", 6)
    x[0, 0] = float("nan")
    y = layer.run(x)
    assert y[0].isnan().all() and y[1].isfinite().all()


def test_empty_runs():
    import torch
    w, b = _layer(32, 128, 5, False)
    layer = sp.Fp8Linear.from_dense(w, b)
    assert layer.run(torch.empty((0, 128), device=device())).shape == (0, 32)
    q, s = sp.quantize_fp8(torch.empty((0, 128), device=device()))
    assert q.shape == (0, 128) and s.shape == (1, 0)


def test_linear_on_another_stream_and_in_a_graph():
    """The caller's stream carries all of a call's work; a recorded call replays."""
    import torch
    w, b = _layer(512, 1024, 8, True)
    layer = sp.Fp8Linear.from_dense(w, b)
    x = _rows(100, 1024, "bf16", 2)
    y = torch.empty((100, 512), dtype=torch.bfloat16, device=device())
    space = torch.empty(layer.workspace_bytes(100, torch.bfloat16), dtype=torch.uint8, device=device())
    ref = layer.run(x).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer.run(x, y=y, workspace=space, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(x, y=y, workspace=space)
    for k in range(3):
        x.copy_(_rows(100, 1024, "bf16", 20 + k))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, layer.run(x)), "replay %d" % k
