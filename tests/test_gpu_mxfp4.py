"""The 4-bit form and dense layers with it, against 64 bits."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import act_ref, torch_dtype
from gpu_util import device, note
from serve_util import lines, linear4_tol, packed, quantize4_ref, to_numpy, unpacked, values4

pytestmark = pytest.mark.gpu


def _draw(rows, cols, dtype, seed, stride=None):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols if stride is None else stride), generator=g)
    x[:, :: 37] *= 30
    return x.to(torch_dtype(dtype)).to(device())[:, :cols]


def _codes(x):
    q, s = sp.quantize_mxfp4(x)
    return unpacked(q.cpu().numpy(), s.cpu().numpy())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (2, 32), (9, 33), (8, 255), (7, 256), (5, 257), (16, 1280),
                                       (100, 1000), (1, 8192), (2100, 520), (33, 40000)])
def test_quantizer(rows, cols, dtype):
    note("quantize4 %d x %d %s" % (rows, cols, dtype))
    for stride in (cols, cols + 3, cols + 8):
        x = _draw(rows, cols, dtype, 1, stride)
        q, s = sp.quantize_mxfp4(x)
        ref = packed(*quantize4_ref(to_numpy(x)))
        assert np.array_equal(q.cpu().numpy(), ref[0]) and np.array_equal(s.cpu().numpy(), ref[1])


def test_quantizer_of_every_half_value():
    """All float16 values that are finite, each block led by another magnitude; then as bfloat16 bits."""
    import torch
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    for kind in (torch.float16, torch.bfloat16):
        v = bits.view(kind)
        v = v[torch.isfinite(v)]
        lead = v[torch.randperm(len(v), generator=torch.Generator().manual_seed(3))]
        x = torch.zeros((len(v) // 31, 32), dtype=kind)
        x[:, :31] = v[:len(v) // 31 * 31].view(-1, 31)
        x[:, 31] = lead[:len(x)]
        code, scale = _codes(x.to(device()))
        ref = quantize4_ref(to_numpy(x))
        assert np.array_equal(scale, ref[1]) and np.array_equal(code, ref[0])


def test_quantizer_of_borders_and_lost_blocks():
    import torch
    x = torch.zeros((3, 512))
    x[0, 0], x[0, 1] = 6.0, -0.0
    x[0, 2:16] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0])
    x[0, 32], x[0, 64], x[0, 96] = 6.9999995, 7.0, -3.5
    x[1, 0], x[1, 32], x[1, 64], x[1, 96:128] = float("inf"), float("nan"), float("-inf"), 2.0 ** -149
    x[1, 1], x[1, 33] = 5.0, -5.0
    x[2, 0], x[2, 32], x[2, 64], x[2, 96] = 3.4028234e38, 2.0 ** -126, 2.0 ** -125 * 1.75, 2.0 ** -128
    code, scale = _codes(x.to(device()))
    ref = quantize4_ref(to_numpy(x))
    assert np.array_equal(scale, ref[1]) and np.array_equal(code, ref[0])
    assert scale[1, :3].tolist() == [255, 255, 255] and (code[1, :96] == 0).all()


def _layer(cout, cin, seed, bias=True, act="none"):
    import torch
    g = torch.Generator().manual_seed(seed)
    w = torch.randn((cout, cin), generator=g).to(device()) / cin ** 0.5
    b = torch.randn(cout, generator=g).to(device()) if bias else None
    return sp.Mxfp4Linear.from_dense(w, b, act)


def _weight_values(layer):
    return values4(*unpacked(layer.w.cpu().numpy(), layer.w_scale.cpu().numpy()), layer.cin)


def _check(layer, x, y, dtype):
    xv, wv = values4(*quantize4_ref(to_numpy(x)), layer.cin), _weight_values(layer)
    b = 0.0 if layer.bias is None else layer.bias.cpu().double().numpy()
    ref = act_ref(xv @ wv.T + b, layer.act)
    tol = linear4_tol(ref, np.abs(xv) @ np.abs(wv).T + np.abs(b), layer.cin, dtype)
    err = np.abs(to_numpy(y) - ref)
    assert (err <= tol).all(), (err / tol).max()


SIZES = [(1, 1, 1), (1, 64, 10), (2, 300, 17), (3, 1000, 64), (1, 4096, 4096), (1, 5000, 100), (8, 2048, 300), (16, 256, 1000),
         (17, 512, 130), (31, 1280, 960), (32, 4096, 512), (33, 640, 200), (64, 1024, 1024), (65, 257, 65), (100, 8192, 128),
         (128, 3000, 260), (200, 768, 3001), (257, 500, 513), (500, 1024, 256), (300, 4096, 640), (777, 1000, 2500)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cin,cout", SIZES)
def test_linear(n, cin, cout, dtype):
    note("linear4 %d x %d -> %d %s" % (n, cin, cout, dtype))
    layer = _layer(cout, cin, 1, n % 2 == 1, ("none", "relu", "relu6")[n % 3])
    x = _draw(n, cin, dtype, 2)
    _check(layer, x, layer.run(x), dtype)


@pytest.mark.parametrize("n,cin,cout,dtype", [(9, 2300, 33, "bf16"), (3, 1000, 5000, "f32"), (8, 500, 4100, "f16"), (13, 300, 70000, "f16"),
                                              (20, 300, 9000, "bf16"), (50, 300, 33000, "bf16"), (300, 600, 2048, "f32"),
                                              (300, 4200, 4096, "bf16"), (290, 500, 4100, "f16"), (1200, 2100, 4000, "bf16"),
                                              (1200, 300, 4001, "f16"), (2600, 300, 4100, "bf16"), (2600, 513, 4096, "f32")])
def test_linear_of_every_tile(n, cin, cout, dtype):
    note("linear4 %d x %d -> %d %s" % (n, cin, cout, dtype))
    layer = _layer(cout, cin, 3, True, "relu6" if n % 2 else "none")
    x = _draw(n, cin, dtype, 4)
    _check(layer, x, layer.run(x), dtype)


@pytest.mark.parametrize("n,cin,cout", [(1, 1024, 100), (20, 2048, 333), (40, 512, 512), (130, 1536, 264), (600, 1024, 520),
                                        (1100, 512, 1030), (64, 16384, 128), (2100, 256, 2050)])
def test_exact_sums(n, cin, cout):
    """With scales of 1 and codes at random every sum is a multiple of 1/4 below 2^22: exact, whatever its order."""
    import torch
    note("exact %d x %d -> %d" % (n, cin, cout))
    g = torch.Generator().manual_seed(n)
    w, x = (torch.randint(0, 256, (r, lines(cin) * 128), generator=g, dtype=torch.uint8) for r in (cout, n))
    ones = [torch.full((lines(cin), r, 8), 127, dtype=torch.uint8, device=device()) for r in (cout, n)]
    layer = sp.Mxfp4Linear(w.to(device()), ones[0], cout, lines(cin) * 256)
    y = layer.run(x.to(device()), ones[1], dtype=torch.float32)
    ref = values4(*unpacked(x.numpy(), ones[1].cpu().numpy()), layer.cin) @ _weight_values(layer).T
    assert np.array_equal(y.cpu().double().numpy(), ref)


@pytest.mark.parametrize("n", [3, 40, 300])
def test_scales_of_every_block_count(n):
    """One block's scale differs at a time: its place in rows, lines and halves is the right one."""
    import torch
    note("scales %d" % n)
    cin, cout = 768, 130
    g = torch.Generator().manual_seed(5)
    w = torch.randint(0, 256, (cout, 384), generator=g, dtype=torch.uint8).to(device())
    x = torch.randint(0, 256, (n, 384), generator=g, dtype=torch.uint8).to(device())
    ws = torch.randint(120, 131, (3, cout, 8), generator=g, dtype=torch.uint8).to(device())
    xs = torch.randint(120, 131, (3, n, 8), generator=g, dtype=torch.uint8).to(device())
    layer = sp.Mxfp4Linear(w, ws, cout, cin)
    y = layer.run(x, xs, dtype=torch.float32).cpu().double().numpy()
    xv = values4(*unpacked(x.cpu().numpy(), xs.cpu().numpy()), cin)
    wv = _weight_values(layer)
    ref = xv @ wv.T
    assert (np.abs(y - ref) <= linear4_tol(ref, np.abs(xv) @ np.abs(wv).T, cin, "f32")).all()


@pytest.mark.parametrize("n", [1, 20, 100, 700])
def test_lost_blocks_stay_in_their_row_and_channel(n):
    import torch
    note("lost %d" % n)
    layer = _layer(140, 600, 3, False)
    x = _draw(n, 600, "bf16", 4).clone()
    clean = layer.run(x)
    row = n // 2
    x[row, 599] = float("inf")
    y = layer.run(x)
    assert torch.isnan(y[row]).all()
    keep = torch.arange(n) != row
    assert torch.equal(y[keep], clean[keep])
    layer.w_scale[2, 77, 1] = 255
    y = layer.run(x)
    assert torch.isnan(y[:, 77]).all() and torch.equal(y[keep][:, :77], clean[keep][:, :77])


@pytest.mark.parametrize("n,cin,cout", [(1, 300, 33), (5, 1000, 100), (60, 512, 64), (300, 700, 260)])
def test_strides_outputs_and_workspaces_of_the_caller(n, cin, cout):
    """Strided rows, codes given, y given: the same bits; nothing behind y or the workspace changes."""
    import torch
    layer = _layer(cout, cin, 6)
    wide = _draw(n, cin, "bf16", 7, cin + 5)
    y = layer.run(wide.contiguous())
    assert torch.equal(layer.run(wide), y)
    q, s = sp.quantize_mxfp4(wide)
    assert torch.equal(layer.run(q, s, dtype=torch.bfloat16), y)
    size = layer.workspace_bytes(n, torch.bfloat16)
    space = torch.full((size + 64,), 7, dtype=torch.uint8, device=device())
    out = torch.full((n + 2, cout), 5.0, dtype=torch.bfloat16, device=device())
    layer.run(wide, y=out[:n], workspace=space)
    assert torch.equal(out[:n], y) and (out[n:] == 5).all() and (space[size:] == 7).all()


def test_results_do_not_depend_on_the_call():
    import torch
    layer = _layer(512, 2048, 8)
    for n in (1, 32, 200):
        x = _draw(n, 2048, "f16", 9)
        first = layer.run(x)
        assert all(torch.equal(layer.run(x), first) for _ in range(5))


def test_many_rows():
    """More rows than a grid's second axis has."""
    import torch
    layer = _layer(3, 40, 10)
    x = _draw(1, 40, "f16", 11).repeat(300000, 1)
    y = layer.run(x)
    assert (y == y[0]).all()
    _check(layer, x[:2], y[:2], "f16")


def test_no_rows_and_refusals():
    import torch
    layer = _layer(20, 300, 12)
    assert layer.run(torch.empty((0, 300), device=device())).shape == (0, 20)
    assert sp.quantize_mxfp4(torch.empty((0, 300), device=device()))[1].shape == (2, 0, 8)
    x = torch.zeros((4, 300), device=device())
    q, s = sp.quantize_mxfp4(x)
    for call in (lambda: layer.run(x[:, :299]), lambda: layer.run(x.cpu()), lambda: layer.run(q, s),
                 lambda: layer.run(q, s[:, :3], dtype=torch.float32), lambda: layer.run(x, y=x),
                 lambda: layer.run(q[:, :128], s, dtype=torch.float32), lambda: sp.quantize_mxfp4(x, q[:, :-1]),
                 lambda: sp.quantize_mxfp4(x, q, s.transpose(0, 1)), lambda: sp.Mxfp4Linear(q, s, 4, 600),
                 lambda: sp.Mxfp4Linear(q, s, 4, 300, torch.zeros(3, device=device()))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sp.SpconvError):
        layer.run(torch.zeros((40, 300), device=device()), workspace=torch.empty(16, dtype=torch.uint8, device=device()))
