"""How exactly dense layers sum products of codes, shown where large products
cancel: in 32 bits for results in 32 bits and for few rows, else within what the
8-bit matrix instruction may cut off (fp8_cut.py)."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_cut import cut8
from fp8_util import BLOCK, block_values, blocks, code_values, linear_ref, linear_tol, row_values, torch_dtype
from gpu_util import device, note

pytestmark = pytest.mark.gpu


def _codes(rows, cols, g, pairs, sign, rest):
    """Codes of well spread values; in one group of 8 channels of every
    ``pairs``-th block 448 and sign * 448 and six of ``rest``."""
    import torch
    v = torch.zeros((rows, blocks(cols) * BLOCK))
    v[:, :cols] = torch.randn((rows, cols), generator=g) * 2
    for b in range(0, cols // BLOCK, pairs):
        at = b * BLOCK + 8 * (b * 5 % 16)
        v[:, at:at + 8] = rest
        v[:, at], v[:, at + 1] = 448.0, sign * 448.0
    return v.to(device()).to(torch.float8_e4m3fn)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout", [(4, 128, 130), (20, 300, 64), (40, 128, 130), (70, 700, 200), (300, 2200, 300),
                                        (40, 6200, 64), (600, 128, 3900), (2060, 256, 3600)])
@pytest.mark.parametrize("pairs", [1, 1000])
def test_large_products_that_cancel(dtype, n, cin, cout, pairs):
    import torch
    note("linear %s n %d cin %d cout %d, a pair in every %d blocks" % (dtype, n, cin, cout, pairs))
    g = torch.Generator().manual_seed(n + cin)
    x, w = _codes(n, cin, g, pairs, 1, 1.75), _codes(cout, cin, g, pairs, -1, 3.5)
    xs = (torch.rand((blocks(cin), n), generator=g) + 0.5).to(device()) / 64
    ws = (torch.rand((blocks(cout), blocks(cin)), generator=g) + 0.5).to(device()) / 64
    layer = sp.Fp8Linear(w, ws, cout, cin)
    y = layer.run(x, xs, dtype=torch_dtype(dtype)).double().cpu().numpy()
    xq, xsn, wq, wsn = code_values(x), xs.cpu().numpy(), code_values(w), ws.cpu().numpy()
    ref, terms = linear_ref(row_values(xq, xsn, cin), block_values(wq, wsn, cin), None, "none")
    tol = linear_tol(ref, terms, cin, dtype)
    if dtype != "f32" and n > 32:
        tol = tol + cut8(xq, xsn, wq, wsn)
    err = np.abs(y - ref)
    assert (err <= tol).all(), "worst error / tolerance %.3g" % float((err / tol).max())


@pytest.mark.parametrize("n", [40, 300])
def test_what_is_cut_off_is_of_eight_channels(n):
    """A term beside a pair 448 * 448 - 448 * 448 counts in steps of 8 where a
    16-bit result is summed in 8 bits, and as it is beyond their 8 channels."""
    import torch
    note("linear bf16 n %d, one term beside a pair" % n)
    x = torch.zeros((n, 128))
    w = torch.zeros((4, 128))
    x[:, 0] = x[:, 1] = w[:, 0] = 448.0
    w[:, 1] = -448.0
    x[:, 7], x[:, 8] = 1.75, 1.75
    w[0, 7] = w[1, 8] = 3.5      # 6.125
    w[2, 7] = w[3, 8] = 112.0    # 196
    one = torch.ones((1, n), device=device())
    layer = sp.Fp8Linear(w.to(device()).to(torch.float8_e4m3fn), torch.ones((1, 1), device=device()), 4, 128)
    x = x.to(device()).to(torch.float8_e4m3fn)
    exact = layer.run(x, one, dtype=torch.float32)
    assert torch.equal(exact, torch.tensor([6.125, 6.125, 196.0, 196.0], device=device()).expand(n, 4))
    y = layer.run(x, one, dtype=torch.bfloat16).float()
    assert (y[:, 1] == 6.125).all() and (y[:, 3] == 196.0).all()
    assert ((y[:, 0] - 6.125).abs() < 8).all() and ((y[:, 2] - 196.0).abs() < 8).all()
