"""Norms of rows, with the residual's addition and 8-bit rows, against 64 bits."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import ROUND, torch_dtype
from gpu_util import device, note
from serve_util import norm_ref, norm_tol, to_numpy

pytestmark = pytest.mark.gpu


def _draw(rows, cols, dtype, seed, stride=None, scale=1.0):
    """A matrix with its own row stride, in memory that holds other values between the rows."""
    import torch
    g = torch.Generator().manual_seed(seed)
    stride = cols if stride is None else stride
    x = (torch.randn((rows, stride), generator=g) * scale).to(torch_dtype(dtype)).to(device())
    return x[:, :cols]


def _check(x, gain, residual, y, total, dtype, eps=1e-6):
    ref, h = norm_ref(to_numpy(x), None if residual is None else to_numpy(residual),
                      None if gain is None else to_numpy(gain), eps)
    err = np.abs(to_numpy(y) - ref)
    assert (err <= norm_tol(ref, x.shape[1], dtype)).all(), (err - norm_tol(ref, x.shape[1], dtype)).max()
    if total is not None:
        kind = {"torch.float32": "f32", "torch.float16": "f16", "torch.bfloat16": "bf16"}[str(total.dtype)]
        # one 32-bit addition, one rounding
        assert (np.abs(to_numpy(total) - h) <= np.abs(h) * (2.0 ** -24 + 1.01 * ROUND[kind]) + 2.0 ** -25).all()


SIZES = [(1, 1), (3, 7), (5, 127), (1, 128), (2, 129), (33, 512), (9, 513), (4, 1000), (1, 1280), (300, 2048), (7, 2049),
         (3, 4100), (2, 8192), (1, 8200), (3, 32768), (2, 32769), (1, 100003)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rows(rows, cols, dtype):
    note("norm %d x %d %s" % (rows, cols, dtype))
    x, gain = _draw(rows, cols, dtype, 1), _draw(1, cols, dtype, 2)[0]
    _check(x, gain, None, sp.rms_norm(x, gain), None, dtype)
    _check(x, None, None, sp.rms_norm(x, None, 0.5), None, dtype, 0.5)


@pytest.mark.parametrize("dtype,of_r,of_g,of_y", [("f32", "f32", "f32", "f32"), ("f16", "f16", "f16", "f16"),
                                                  ("f16", "f32", "f16", "f32"), ("bf16", "bf16", "f32", "bf16"),
                                                  ("bf16", "f32", "bf16", "f32"), ("bf16", "bf16", "bf16", "f32")])
@pytest.mark.parametrize("rows,cols", [(1, 1280), (5, 127), (70, 512), (3, 1001), (9, 4096), (2, 33000)])
def test_residuals_and_types(rows, cols, dtype, of_r, of_g, of_y):
    note("norm %d x %d %s %s %s %s" % (rows, cols, dtype, of_r, of_g, of_y))
    x, r = _draw(rows, cols, dtype, 3), _draw(rows, cols, of_r, 4, scale=3.0)
    gain = _draw(1, cols, of_g, 5)[0]
    y, total = sp.rms_norm(x, gain, residual=r, dtype=torch_dtype(of_y))
    assert y.dtype == torch_dtype(of_y) and total.dtype == torch_dtype(of_r)
    _check(x, gain, r, y, total, of_y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1000, 1024, 33000])
def test_strides_leave_the_rest_alone(cols, dtype):
    """Rows inside wider ones, at every alignment that an odd stride gives."""
    import torch
    for stride in (cols, cols + 1, cols + 24):
        x, r = _draw(6, cols, dtype, 6, stride), _draw(6, cols, dtype, 7, stride + 8)
        gain = _draw(1, cols, dtype, 8)[0]
        wide = [torch.full((6, stride + extra), 77.0, dtype=torch_dtype(dtype), device=device()) for extra in (0, 3)]
        y, total = sp.rms_norm(x, gain, residual=r, y=wide[0][:, :cols], total=wide[1][:, :cols])
        _check(x, gain, r, y, total, dtype)
        assert all((w[:, cols:] == 77).all() for w in wide)


@pytest.mark.parametrize("cols", [64, 1280, 5000, 40000])
def test_in_place_equals_apart(cols):
    import torch
    x, r, gain = _draw(5, cols, "bf16", 9), _draw(5, cols, "bf16", 10), _draw(1, cols, "bf16", 11)[0]
    y, total = sp.rms_norm(x, gain, residual=r)
    for t_at, y_at in (("r", "x"), ("x", "r"), ("r", None), (None, "x"), ("x", None)):
        xs, rs = x.clone(), r.clone()
        place = {"x": xs, "r": rs, None: None}
        y2, total2 = sp.rms_norm(xs, gain, residual=rs, y=place[y_at], total=place[t_at])
        assert torch.equal(y2, y) and torch.equal(total2, total), (t_at, y_at)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 100), (17, 128), (5, 130), (40, 1000), (3, 4096), (300, 640), (2, 9000), (2, 33000)])
@pytest.mark.parametrize("residual", [False, True])
def test_8_bit_rows_are_those_of_the_32_bit_ones(rows, cols, dtype, residual):
    """rms_norm_fp8 = quantize_fp8 of the norm in float32, bit for bit; y beside it, too."""
    import torch
    note("norm fp8 %d x %d %s %s" % (rows, cols, dtype, residual))
    x, gain = _draw(rows, cols, dtype, 12), _draw(1, cols, dtype, 13)[0]
    r = _draw(rows, cols, dtype, 14) if residual else None
    wide = sp.rms_norm(x, gain, residual=r, dtype=torch.float32)
    wide = wide[0] if residual else wide
    y = torch.empty_like(x)
    got = sp.rms_norm_fp8(x, gain, residual=r, y=y)
    q, scale = sp.quantize_fp8(wide)
    assert torch.equal(got[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(got[1], scale)
    assert torch.equal(y, wide.to(x.dtype))
    assert len(got) == (3 if residual else 2)


def test_rows_do_not_touch_each_other():
    """An infinity, a NaN, zeros and huge values: each row's result is its own."""
    import torch
    x = _draw(6, 1024, "f32", 15).clone()
    x[1, 5], x[2, 1000], x[3], x[4] = float("inf"), float("nan"), 0.0, 1e20
    y = sp.rms_norm(x)
    q, scale = sp.rms_norm_fp8(x)
    for row in (0, 5):
        assert torch.equal(y[row:row + 1], sp.rms_norm(x[row:row + 1].clone()))
    assert torch.isnan(y[1, 5]) and (y[1, :5] == 0).all() and torch.isnan(y[2]).all()
    assert (y[3] == 0).all() and (y[4] == 0).all()  # the sum of 1e40 is infinite
    assert torch.isnan(scale[:, 2]).all() and torch.isnan(scale[0, 1]) and not torch.isnan(scale[1:, 1]).any()
    assert torch.isnan(sp.rms_norm(x[3:4], eps=0.0)).all()  # 0 / 0


def test_no_rows():
    import torch
    x = torch.empty((0, 64), device=device())
    assert sp.rms_norm(x).shape == (0, 64)
    q, scale, total = sp.rms_norm_fp8(x, residual=x)
    assert q.shape == (0, 128) and scale.shape == (1, 0) and total.shape == (0, 64)
    assert sp.rms_norm(torch.empty((3, 0), device=device())).shape == (3, 0)


@pytest.mark.parametrize("cols", [4096, 40000])
def test_rows_past_32_bit_offsets(cols):
    """Rows of one buffer whose ends lie 5 GB apart."""
    import torch
    x = torch.empty((2, 1 << 31), dtype=torch.bfloat16, device=device())[:, :cols]
    x.copy_(_draw(2, cols, "bf16", 16))
    near = x.contiguous()
    y = torch.empty((2, 1 << 30), dtype=torch.float32, device=device())[:, :cols]
    sp.rms_norm(x, y=y)
    assert torch.equal(y.contiguous(), sp.rms_norm(near, dtype=torch.float32))


def test_refusals():
    import torch
    x = torch.zeros((4, 256), device=device())
    for call in (lambda: sp.rms_norm(x[:, ::2]), lambda: sp.rms_norm(x, torch.zeros(255, device=device())),
                 lambda: sp.rms_norm(x, torch.zeros(256)), lambda: sp.rms_norm(x, residual=x[:3]),
                 lambda: sp.rms_norm(x, residual=x.cpu()), lambda: sp.rms_norm(x, total=x),
                 lambda: sp.rms_norm(x, y=x[:, :255]), lambda: sp.rms_norm(x, y=x.clone().half(), dtype=torch.float32),
                 lambda: sp.rms_norm(x, residual=x, total=x.half()), lambda: sp.rms_norm_fp8(x, q=x),
                 lambda: sp.rms_norm(x.T), lambda: sp.rms_norm_fp8(x, scale=torch.zeros((4, 2), device=device()))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(sp.SpconvError):
        sp.rms_norm(x, eps=-1.0)
    with pytest.raises(sp.SpconvError):  # x itself takes either, not both
        sp.rms_norm(x, residual=x.clone(), y=x, total=x)
    with pytest.raises(sp.SpconvError):
        sp.rms_norm(x, dtype=torch.bfloat16)
