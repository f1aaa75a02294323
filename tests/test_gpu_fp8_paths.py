"""Quantiser and dense layers at the sizes that choose each way to load and store:
several blocks of a row at once, and every tile shape's vector epilogue."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_cut import cut8
from fp8_util import (block_values, code_values, linear_ref, linear_tol, quantize_ref, row_values,
                      torch_dtype)
from gpu_util import device, note

pytestmark = pytest.mark.gpu


def _rows(rows, cols, dtype, seed, extra=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn((rows, cols + extra), generator=g).to(torch_dtype(dtype)).to(device())[:, :cols]


# 4096 and more groups of 16 rows and blocks: four blocks of a row at once, the last ones part of a row's end
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,extra", [(2000, 4300, 0), (1030, 8192, 4), (5001, 1793, 3)])
def test_quantize_several_blocks_at_once(dtype, rows, cols, extra):
    note("quantize %s %d x %d + %d" % (dtype, rows, cols, extra))
    x = _rows(rows, cols, dtype, rows, extra)
    q, scale = sp.quantize_fp8(x)
    ref_q, ref_s = quantize_ref(x.float().cpu().numpy(), 1)
    assert np.array_equal(scale.cpu().numpy(), ref_s)
    assert np.array_equal(code_values(q), ref_q)


# cout a multiple of 8 (whole lines of 16-bit results), of 4 (whole vectors), rows that end inside a tile;
# tiles of 256 x 256, then 128 x 128 and 128 x 64 in both depths
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout,act", [(4099, 384, 3080, "none"), (4099, 300, 3076, "relu"), (2050, 256, 2056, "none"),
                                            (1500, 384, 1544, "relu6"), (1000, 2176, 1032, "none"), (500, 640, 2564, "none"),
                                            (300, 2304, 1608, "relu"), (100, 4200, 264, "none"), (60, 520, 30008, "none")])
def test_linear_vector_epilogues(dtype, n, cin, cout, act):
    import torch
    note("linear %s n %d cin %d cout %d" % (dtype, n, cin, cout))
    g = torch.Generator().manual_seed(cin)
    w = (torch.randn((cout, cin), generator=g) / cin ** 0.5).to(device())
    bias = torch.randn(cout, generator=g).to(device())
    layer = sp.Fp8Linear.from_dense(w, bias, act)
    x = _rows(n, cin, dtype, n)
    y = layer.run(x)
    q, s = quantize_ref(x.float().cpu().numpy(), 1)
    wq, ws = code_values(layer.w), layer.w_scale.cpu().numpy()
    ref, terms = linear_ref(row_values(q, s, cin), block_values(wq, ws, cin), bias.cpu().numpy(), act)
    tol = linear_tol(ref, terms, cin, dtype)
    if dtype != "f32":
        tol = tol + cut8(q, s, wq, ws)
    err = np.abs(y.double().cpu().numpy() - ref)
    assert y.dtype == torch_dtype(dtype) and (err <= tol).all(), "worst error / tolerance %.3g" % float((err / tol).max())
    # together: sums on the 8-bit instruction 5e-5 of well spread values, in 32 bits 2e-6, and one rounding
    off = {"f32": 2e-6, "f16": 5e-5 + 2.0 ** -11 / 3 ** 0.5, "bf16": 5e-5 + 2.0 ** -8 / 3 ** 0.5}[dtype]
    assert np.linalg.norm(err) <= off * np.linalg.norm(ref)
