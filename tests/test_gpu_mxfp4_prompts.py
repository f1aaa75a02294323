"""The 4-bit quantiser's kernel for large matrices, and products held to their own roundings."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import act_ref, torch_dtype
from gpu_util import device, note
from serve_bounds import linear4_tight
from serve_util import packed, quantize4_ref, to_numpy, unpacked, values4

pytestmark = pytest.mark.gpu


def _draw(rows, cols, dtype, seed, extra=0):
    """A matrix whose rows lie `extra` values apart, some columns larger and some blocks zero."""
    import torch
    g = torch.Generator(device()).manual_seed(seed)
    x = torch.randn((rows, cols + extra), generator=g, device=device())
    x[:, ::37] *= 30
    x[1::5, :40] = 0
    return x.to(torch_dtype(dtype))[:, :cols]


def _by_parts(x, rows):
    """The same from calls of so few rows that they take the kernel for small matrices."""
    import torch
    parts = [sp.quantize_mxfp4(x[i:i + rows]) for i in range(0, len(x), rows)]
    return torch.cat([q for q, _ in parts]), torch.cat([s for _, s in parts], dim=1)


# 4096 groups of 8 rows and a line of 256 columns take four lines a thread: of 1 to 9 lines, just below, at and above
LARGE = [(32768, 200), (32760, 256), (16400, 512), (10950, 700), (8200, 1024), (8192, 1000), (8184, 1024), (6600, 1100), (5470, 1500),
         (4700, 1792), (4097, 2000), (3650, 2300), (1000, 8400), (2049, 4096)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", LARGE)
def test_large_matrices(rows, cols, dtype):
    """Bit for bit those of small calls, and of the definition where rows are looked at."""
    import torch
    note("quantize4 %d x %d %s" % (rows, cols, dtype))
    for extra in (0, 1, 8):
        x = _draw(rows, cols, dtype, 1, extra)
        q, s = sp.quantize_mxfp4(x)
        small = _by_parts(x, 8 * (4095 // -(-cols // 256)))
        assert torch.equal(q, small[0]) and torch.equal(s, small[1])
        some = torch.cat([torch.arange(9), torch.arange(rows - 9, rows), torch.randperm(rows, generator=torch.Generator().manual_seed(2))[:40]]).to(device())
        ref = packed(*quantize4_ref(to_numpy(x[some])))
        assert np.array_equal(q[some].cpu().numpy(), ref[0]) and np.array_equal(s[:, some].cpu().numpy(), ref[1])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_matrices_with_lost_blocks(dtype):
    """An infinity or a NaN loses its block and no other; nothing behind the outputs changes."""
    import torch
    rows, cols = 4200, 2010
    note("quantize4 lost %s" % dtype)
    x = _draw(rows, cols, dtype, 3)
    clean = sp.quantize_mxfp4(x)
    x = x.clone()
    x[7, 5], x[4199, 2009], x[100, 1024] = float("inf"), float("nan"), float("-inf")
    q, s = torch.full((rows + 1, 1024), 9, dtype=torch.uint8, device=device()), torch.full((8 * rows * 8 + 16,), 9, dtype=torch.uint8, device=device())
    sp.quantize_mxfp4(x, q[:rows], s[:8 * rows * 8].view(8, rows, 8))
    codes, scales = clean[0].clone(), clean[1].clone()
    for row, col in ((7, 5), (4199, 2009), (100, 1024)):
        codes[row, col // 32 * 16:col // 32 * 16 + 16] = 0
        scales[col // 256, row, col % 256 // 32] = 255
    assert torch.equal(q[:rows], codes) and torch.equal(s[:8 * rows * 8].view(8, rows, 8), scales)
    assert bool((q[rows:] == 9).all()) and bool((s[8 * rows * 8:] == 9).all())


# every kernel: rows quantised inside, codes without tiles, each tile, one and two groups of wavefronts
PRODUCTS = [(1, 100, 40), (1, 4096, 500), (3, 1000, 5000), (8, 500, 4100), (9, 2300, 33), (13, 300, 70000), (16, 256, 1000), (17, 200, 130),
            (64, 1024, 1024), (100, 8192, 128), (20, 300, 9000), (50, 300, 33000), (300, 600, 2048), (300, 4200, 4096), (290, 250, 4100),
            (1200, 2100, 4000), (1200, 256, 4001), (2600, 300, 4100), (2600, 513, 4096)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout", PRODUCTS)
def test_products(n, cin, cout, dtype):
    import torch
    note("linear4 %d x %d -> %d %s" % (n, cin, cout, dtype))
    g = torch.Generator(device()).manual_seed(4)
    act = ("none", "relu", "relu6")[n % 3]
    layer = sp.Mxfp4Linear.from_dense(torch.randn((cout, cin), generator=g, device=device()) / cin ** 0.5,
                                      torch.randn(cout, generator=g, device=device()) if n % 2 else None, act)
    x = _draw(n, cin, dtype, 5)
    y = layer.run(x)
    xv = values4(*quantize4_ref(to_numpy(x)), cin)
    wv = values4(*unpacked(layer.w.cpu().numpy(), layer.w_scale.cpu().numpy()), cin)
    b = 0.0 if layer.bias is None else layer.bias.cpu().double().numpy()
    ref = act_ref(xv @ wv.T + b, act)
    off = np.abs(to_numpy(y) - ref) / linear4_tight(ref, np.abs(xv) @ np.abs(wv).T + np.abs(b), cin, dtype)
    assert off.max() <= 1, off.max()
