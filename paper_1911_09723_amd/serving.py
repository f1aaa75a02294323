"""Norms, dense layers in 4 bits and sampling, for torch tensors.

The arithmetic runs in libspconv's kernels (include/spconv.h says what each
computes and how its arrays are laid out); this module checks shapes, types and
strides, allocates what a call writes with torch's allocator and passes
addresses on, as ``experts.py`` does.  What that module says about streams and
gradients holds here, too.
"""

from __future__ import annotations

from functools import lru_cache

from . import experts as _experts
from .experts import BLOCK, _bytes, _given, _gpu_of, _handle, _matrix, _type
from .spconv import _ACTS, F32, MXFP4, _check, spconv_linear_mxfp4_workspace, spconv_sample_workspace

LINE = 256
# sizes are asked for on every call
_linear_workspace = lru_cache(maxsize=1024)(spconv_linear_mxfp4_workspace)
_sample_workspace = lru_cache(maxsize=1024)(spconv_sample_workspace)


def _lines(n: int) -> int:
    return -(-n // LINE)


def _rows_like(t, shape, device, what: str) -> int:
    """The row stride of t, checked to be a matrix of this shape with contiguous rows on this device."""
    rows, cols = shape
    if t.shape != shape or t.get_device() != device:
        raise ValueError("%s must be a matrix [%d, %d] on GPU %d" % (what, rows, cols, device))
    ld, step = t.stride()
    if (step != 1 and cols > 1) or (rows > 1 and ld < cols):
        raise ValueError("%s must have contiguous rows" % what)
    return ld if rows > 1 else cols


def _norm(x, gain, eps, residual, total, y, dtype, q, scale, stream):
    """Queue the norm of x into the outputs given, and into y of `dtype` (x's where None) and total,
    which are made here where neither y nor q, or a residual without total, is given; returns (y, total)."""
    kind = _type(x.dtype, "x")
    rows, cols, ldx, device = _matrix(x, "x")
    shape, like = (rows, cols), _experts._torch.empty_like  # (rows that lie as x's: contiguous)
    kind_r = kind_g = kind_y = F32
    at_r = at_t = at_g = at_y = None
    ldr = ldt = ldy = cols
    if residual is not None:
        ldr, kind_r, at_r = _rows_like(residual, shape, device, "residual"), _type(residual.dtype, "residual"), residual.data_ptr()
        if total is None:
            total = like(residual)
        elif total.dtype != residual.dtype:
            raise ValueError("total must have the residual's type")
        else:
            ldt = _rows_like(total, shape, device, "total")
        at_t = total.data_ptr()
    elif total is not None:
        raise ValueError("total is the sum with a residual")
    if gain is not None:
        kind_g, at_g = _type(gain.dtype, "gain"), gain.data_ptr()
        if gain.shape != (cols,) or gain.get_device() != device or not gain.is_contiguous():
            raise ValueError("gain must be a contiguous vector of %d values on GPU %d" % (cols, device))
    if y is not None:
        ldy, kind_y = _rows_like(y, shape, device, "y"), _type(y.dtype, "y")
    elif q is None:
        y, kind_y = (like(x), kind) if dtype is None else (like(x, dtype=dtype), _type(dtype, "dtype"))
    if y is not None:
        at_y = y.data_ptr()
    if rows and cols:
        _check(_experts._lib.spconv_rms_norm(
            x.data_ptr(), kind, ldx, at_r, kind_r, ldr, at_t, ldt, at_g, kind_g, eps, at_y, kind_y, ldy,
            None if q is None else q.data_ptr(), None if scale is None else scale.data_ptr(), rows, cols,
            _handle(stream, device)))
    return y, total


def rms_norm(x, gain=None, eps: float = 1e-6, residual=None, y=None, dtype=None, total=None, stream=None):
    """y = h / sqrt(mean(h^2) + eps) * gain over the rows of h = x + residual
    (or x): a matrix [rows, cols] of ``dtype`` (x's, or float32).  With a residual
    the pair (y, total): total is h in the residual's type, into ``total`` (a new
    tensor, or the residual itself) where given."""
    if y is not None and dtype is not None and y.dtype != dtype:
        raise ValueError("y must be of dtype")
    pair = _norm(x, gain, eps, residual, total, y, dtype, None, None, stream)
    return pair[0] if residual is None else pair


def rms_norm_fp8(x, gain=None, eps: float = 1e-6, residual=None, q=None, scale=None, y=None, total=None, stream=None):
    """The same as 8-bit codes [rows, 128 kb] and scales [kb, rows] (kb = ceil(cols /
    128)), as quantize_fp8 makes them of the 32-bit y, for Fp8Linear.run: the pair
    (q, scale), or with a residual (q, scale, total).  ``y``: a matrix that takes
    the unquantised rows, too."""
    _type(x.dtype, "x")
    rows, cols, _, _ = _matrix(x, "x")
    kb, torch = -(-cols // BLOCK), _experts._torch
    if q is None:
        q = x.new_empty((rows, kb * BLOCK), dtype=torch.float8_e4m3fn)
    else:
        _given(q, (rows, kb * BLOCK), torch.float8_e4m3fn, x.device, "q")
    if scale is None:
        scale = x.new_empty((kb, rows), dtype=torch.float32)
    else:
        _given(scale, (kb, rows), torch.float32, x.device, "scale")
    _, total = _norm(x, gain, eps, residual, total, y, None, q, scale, stream)
    return (q, scale) if residual is None else (q, scale, total)


def quantize_mxfp4(x, q=None, scale=None, stream=None):
    """A matrix [rows, cols] as 4-bit codes, two a byte, [rows, 128 lines] (uint8, lines
    = ceil(cols / 256)) and the exponents of a power of two for each 32 columns, plus
    127, [lines, rows, 8] (uint8); rows and weights alike."""
    kind = _type(x.dtype, "x")
    rows, cols, ld, device = _matrix(x, "x")
    lines, torch = -(-cols // LINE), _experts._torch
    if q is None:
        q = x.new_empty((rows, lines * 128), dtype=torch.uint8)
    else:
        _given(q, (rows, lines * 128), torch.uint8, x.device, "q")
    if scale is None:
        scale = x.new_empty((lines, rows, 8), dtype=torch.uint8)
    else:
        _given(scale, (lines, rows, 8), torch.uint8, x.device, "scale")
    if rows and cols:
        _check(_experts._lib.spconv_quantize_mxfp4(x.data_ptr(), kind, ld, rows, cols, q.data_ptr(), scale.data_ptr(),
                                                   _handle(stream, device)))
    return q, scale


class Mxfp4Linear:
    """A dense layer y = act(x W^T + b) with W [cout, cin] in 4 bits:
    ``quantize_mxfp4(W)``'s codes and scales.  It keeps the tensors given."""

    def __init__(self, w, w_scale, cout: int, cin: int, bias=None, act: str = "none"):
        import torch
        if act not in ("none", "relu", "relu6"):
            raise ValueError("act must be 'none', 'relu' or 'relu6'")
        lines, dev = _lines(cin), _gpu_of(w, "w")
        self.w = _given(w, (cout, lines * 128), torch.uint8, dev, "w")
        self.w_scale = _given(w_scale, (lines, cout, 8), torch.uint8, dev, "w_scale")
        self.bias = None if bias is None else _given(bias, (cout,), torch.float32, dev, "bias")
        self.cout, self.cin, self.act, self.device = int(cout), int(cin), act, dev

    @classmethod
    def from_dense(cls, weight, bias=None, act: str = "none"):
        """The layer of a weight [cout, cin] in float32, float16 or bfloat16."""
        w, scale = quantize_mxfp4(weight)
        return cls(w, scale, weight.shape[0], weight.shape[1], bias, act)

    def workspace_bytes(self, n: int, dtype) -> int:
        """Workspace of run() for n rows of a torch dtype that is not quantised yet."""
        return _linear_workspace(_type(dtype, "x"), n, self.cin, self.cout)

    def run(self, x, x_scale=None, y=None, dtype=None, workspace=None, stream=None):
        """y [n, cout] for x [n, cin], or for quantize_mxfp4's codes and scales
        (then ``dtype`` or ``y`` gives y's type; it is x's otherwise)."""
        if x_scale is None:
            kind = _type(x.dtype, "x")
            n, cols, ld, device = _matrix(x, "x")
            if cols != self.cin or device != self.device.index:
                raise ValueError("x must have %d channels and be on %s" % (self.cin, self.device))
            dtype = dtype or (x.dtype if y is None else y.dtype)
        else:
            n, kind, ld, device = int(x.shape[0]), MXFP4, 0, self.device.index
            if _experts._torch is None:
                _experts._bind()
            if device != _experts._device():
                raise ValueError("the layer must be on the current GPU")
            uint8 = _experts._torch.uint8
            _given(x, (n, _lines(self.cin) * 128), uint8, self.device, "x")
            _given(x_scale, (_lines(self.cin), n, 8), uint8, self.device, "x_scale")
            if dtype is None and y is None:
                raise ValueError("quantised rows need y or its dtype")
            dtype = dtype or y.dtype
        if y is None:
            y = x.new_empty((n, self.cout), dtype=dtype)
        else:
            _given(y, (n, self.cout), dtype, self.device, "y")
        size = _linear_workspace(kind, n, self.cin, self.cout)
        space = None
        if size:
            if workspace is None:
                workspace = x.new_empty(size, dtype=_experts._torch.uint8)
            else:
                size = _bytes(workspace, self.device)
            space = workspace.data_ptr()
        if n:
            _check(_experts._lib.spconv_linear_mxfp4(
                x.data_ptr(), kind, ld, None if x_scale is None else x_scale.data_ptr(), self.w.data_ptr(),
                self.w_scale.data_ptr(), None if self.bias is None else self.bias.data_ptr(), _ACTS[self.act],
                y.data_ptr(), _type(dtype, "y"), n, self.cin, self.cout, space, size, _handle(stream, device)))
        return y


def _column(p, n: int, dtype, device, what: str):
    """(address, value) of a parameter: a tensor with a value for each row, or a number for all."""
    if isinstance(p, (int, float)):
        if dtype is _experts._torch.int32 and not -2 ** 31 <= p < 2 ** 31:
            raise ValueError("%s must be a number of 32 bits" % what)
        return None, p
    if p.dtype != dtype or p.shape != (n,) or p.get_device() != device or not p.is_contiguous():
        raise ValueError("%s must be a number or a contiguous %s tensor of %d values on GPU %d" % (what, dtype, n, device))
    return p.data_ptr(), 0


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, ids=None, workspace=None, stream=None):
    """The next token (int32 [n], -1 for a row without any) of each row of logits
    [n, vocab], from random numbers u [n] (float32 in [0, 1)); spconv_sample in
    include/spconv.h defines it.  temperature, top_p and min_p are numbers or
    float32 tensors [n], top_k is a number or an int32 tensor [n]."""
    kind = _type(logits.dtype, "logits")
    n, vocab, ld, device = _matrix(logits, "logits")
    torch = _experts._torch
    f32, i32 = torch.float32, torch.int32
    at_u, _ = _column(u, n, f32, device, "u")
    if at_u is None:
        raise ValueError("u must be a tensor")
    ts, t = _column(temperature, n, f32, device, "temperature")
    ks, k = _column(top_k, n, i32, device, "top_k")
    ps, p = _column(top_p, n, f32, device, "top_p")
    ms, m = _column(min_p, n, f32, device, "min_p")
    if ids is None:
        ids = logits.new_empty((n,), dtype=i32)
    else:
        _given(ids, (n,), i32, logits.device, "ids")
    size = _sample_workspace(kind, n, vocab)
    space = None
    if size:
        if workspace is None:
            workspace = logits.new_empty(size, dtype=torch.uint8)
        else:
            size = _bytes(workspace, logits.device)
        space = workspace.data_ptr()
    _check(_experts._lib.spconv_sample(logits.data_ptr(), kind, ld, at_u, n, vocab, ts, ks, ps, ms, t, k, p, m,
                                       ids.data_ptr(), space, size, _handle(stream, device)))
    return ids
