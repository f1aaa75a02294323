"""Norms of many rows: the kernels with several pieces a thread, calls past the caches, and how exact all of them are."""

import pytest

import paper_1911_09723_amd as sp
from fp8_util import ROUND, torch_dtype
from gpu_util import device, note
from serve_bounds import RMS_ROUND, UNIT, norm64, norm_bound, norm_tight

pytestmark = pytest.mark.gpu

# 512 rows and more take two pieces a thread from 65 pieces on, and calls of 16 MB of x go past the caches:
# of both sides of each rule, whole pieces and not
MANY = [(512, 520), (600, 1000), (513, 1024), (511, 1024), (777, 1032), (520, 2049), (512, 4096), (511, 4096), (512, 4097),
        (700, 8192), (530, 8200)]
PAST = [(16400, 512), (65536, 130), (9000, 1000), (8192, 1024), (4100, 2048), (2100, 4095), (2100, 4096), (1100, 8192), (515, 16384),
        (300, 32761), (300, 32768), (260, 33000)]


def _draw(rows, cols, dtype, seed, extra=0, scale=1.0):
    """A matrix whose rows lie `extra` values apart."""
    import torch
    g = torch.Generator(device()).manual_seed(seed)
    return (torch.randn((rows, cols + extra), generator=g, device=device()) * scale).to(torch_dtype(dtype))[:, :cols]


def _fits(y, ref, cols, dtype, residual):
    off = (y.double() - ref).abs() - norm_tight(ref, cols, dtype, residual)
    assert bool((off <= 0).all()), off.max().item()


def _total_fits(total, h, dtype):
    """One 32-bit sum, one rounding to the type."""
    assert bool(((total.double() - h).abs() <= h.abs() * (UNIT + (0 if dtype == "f32" else ROUND[dtype] * 1.01)) + 2.0 ** -25).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", MANY + PAST)
def test_many_rows(rows, cols, dtype):
    note("norm %d x %d %s" % (rows, cols, dtype))
    x, gain = _draw(rows, cols, dtype, 1), _draw(1, cols, dtype, 2)[0]
    _fits(sp.rms_norm(x, gain), norm64(x, None, gain)[0], cols, dtype, False)


@pytest.mark.parametrize("dtype,of_r,of_g,of_y", [("f32", "f32", "f32", "f32"), ("f16", "f16", "f16", "f16"),
                                                  ("f16", "f32", "f32", "f32"), ("bf16", "bf16", "bf16", "bf16"),
                                                  ("bf16", "f32", "bf16", "f32")])
@pytest.mark.parametrize("rows,cols", MANY[::2] + PAST)
def test_many_rows_with_residual(rows, cols, dtype, of_r, of_g, of_y):
    note("norm %d x %d %s %s %s %s" % (rows, cols, dtype, of_r, of_g, of_y))
    x, r, gain = _draw(rows, cols, dtype, 3), _draw(rows, cols, of_r, 4, scale=3.0), _draw(1, cols, of_g, 5)[0]
    y, total = sp.rms_norm(x, gain, residual=r, dtype=torch_dtype(of_y))
    ref, h = norm64(x, r, gain)
    _fits(y, ref, cols, of_y, True)
    _total_fits(total, h, of_r)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(600, 1000), (520, 4096), (530, 7000), (9000, 1000), (4100, 2048), (2100, 4095), (1100, 8000), (260, 33000)])
def test_strided_rows(rows, cols, dtype):
    """Rows inside wider ones at every alignment: what lies between them stays."""
    import torch
    note("norm %d x %d %s strided" % (rows, cols, dtype))
    gain, kind = _draw(1, cols, dtype, 6)[0], torch_dtype(dtype)
    for extra in (1, 8, 24):
        x, r = _draw(rows, cols, dtype, 7, extra), _draw(rows, cols, dtype, 8, extra + 8)
        wide = [torch.full((rows, cols + extra + more), 77.0, dtype=kind, device=device()) for more in (0, 3)]
        y, total = sp.rms_norm(x, gain, residual=r, y=wide[0][:, :cols], total=wide[1][:, :cols])
        ref, h = norm64(x, r, gain)
        _fits(y, ref, cols, dtype, True)
        _total_fits(total, h, dtype)
        assert all(bool((w[:, cols:] == 77).all()) for w in wide)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(600, 1000), (520, 4096), (530, 8192), (9000, 1000), (4100, 4096), (1100, 8192), (600, 16000), (520, 32768), (260, 33000)])
def test_in_place_equals_apart(rows, cols, dtype):
    import torch
    note("norm %d x %d %s in place" % (rows, cols, dtype))
    x, r, gain = _draw(rows, cols, dtype, 9), _draw(rows, cols, dtype, 10), _draw(1, cols, dtype, 11)[0]
    y, total = sp.rms_norm(x, gain, residual=r)
    for t_at, y_at in (("r", "x"), ("x", "r"), ("r", None), (None, "x")):
        xs, rs = x.clone(), r.clone()
        place = {"x": xs, "r": rs, None: None}
        y2, total2 = sp.rms_norm(xs, gain, residual=rs, y=place[y_at], total=place[t_at])
        assert torch.equal(y2, y) and torch.equal(total2, total), (t_at, y_at)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(600, 1000), (700, 520), (520, 4000), (512, 8100), (9000, 1000), (4100, 2100), (2100, 4096), (1100, 8192), (300, 32700), (260, 33000)])
@pytest.mark.parametrize("residual", [False, True])
def test_8_bit_rows_are_those_of_the_32_bit_ones(rows, cols, dtype, residual):
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


def _e4m3(v):
    """(the nearest e4m3 value, the midpoint that v is nearest to) in 64 bits, |v| up to 448."""
    import torch
    exponent = torch.frexp(v).exponent.clamp(min=-5) - 1
    step = (exponent.long() - 3 + 1023 << 52).view(torch.float64)
    q = torch.round(v / step) * step
    return q, (torch.floor(v / step) + 0.5) * step


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(3, 1280), (600, 1000), (4100, 4096), (260, 33000)])
def test_codes_are_the_definitions_but_for_ties(rows, cols, dtype):
    """A code is another than that of the 64-bit norm only where that lies between two codes, as near to their middle
    as the norm's own roundings, twice (the value's and the largest one's), the factor 448 / a's and the product's are."""
    import torch
    note("codes %d x %d %s" % (rows, cols, dtype))
    x, r, gain = _draw(rows, cols, dtype, 15), _draw(rows, cols, dtype, 16), _draw(1, cols, dtype, 17)[0]
    q, scale, _ = sp.rms_norm_fp8(x, gain, residual=r)
    y, _ = norm64(x, r, gain)
    kb = -(-cols // 128)
    v = torch.zeros((rows, kb * 128), dtype=torch.float64, device=device())
    v[:, :cols] = y
    most = v.view(rows, kb, 128).abs().amax(dim=2)
    bound = norm_bound(cols, True)
    assert bool(((scale.double().T - most / 448).abs() <= most / 448 * (bound + UNIT * 1.01)).all())
    u = (v.view(rows, kb, 128) / most[..., None] * 448).view(rows, -1)
    ref, middle = _e4m3(u)
    other = q.double() != ref
    assert bool(((u - middle).abs()[other] <= u.abs()[other] * (2 * bound + 2 * UNIT * 1.01)).all())


@pytest.mark.parametrize("rows,cols", [(2000, 500), (2000, 1024), (2000, 2048), (3000, 4096), (2000, 8192), (2000, 16384), (1500, 30000), (1500, 33000)])
def test_mean_error(rows, cols):
    """Of rows of all sizes the mean error is that of the two roundings that show: a sum joined, or a root taken, in
    32 bits shows here, though not in the largest error."""
    import torch
    note("mean error %d x %d" % (rows, cols))
    g = torch.Generator(device()).manual_seed(18)
    x = torch.randn((rows, cols), generator=g, device=device()) * 2.0 ** (torch.rand((rows, 1), generator=g, device=device()) * 6 - 3)
    ref, _ = norm64(x)
    off = torch.where(ref == 0, sp.rms_norm(x).double(), (sp.rms_norm(x).double() - ref) / ref)  # (a zero among the draws is exact)
    err = off.square().mean().sqrt().item()
    assert err <= 1.05 * 2 ** 0.5 * RMS_ROUND, err / RMS_ROUND


def test_repeats_of_a_long_call():
    """The same bits in every call, with other calls between."""
    import torch
    x, r, gain = _draw(8192, 4096, "bf16", 19), _draw(8192, 4096, "bf16", 20), _draw(1, 4096, "bf16", 21)[0]
    first = sp.rms_norm_fp8(x, gain, residual=r)
    for _ in range(10):
        sp.rms_norm_fp8(r, gain, residual=x)
        again = sp.rms_norm_fp8(x, gain, residual=r)
        assert torch.equal(first[0].view(torch.uint8), again[0].view(torch.uint8))
        assert all(torch.equal(a, b) for a, b in zip(first[1:], again[1:]))
