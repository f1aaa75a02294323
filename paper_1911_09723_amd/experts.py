"""Dense layers in 8 bits, routers and experts, for torch tensors.

The arithmetic runs in libspconv's kernels (include/spconv.h says what each
computes and how its arrays are laid out); this module checks shapes, types and
strides, allocates what a call writes with torch's allocator (on the current
stream, so that it is reused in order) and passes addresses on.

Work is queued on ``stream`` (a torch stream; default: torch's current one).
With another stream than the current one pass the outputs and the workspace
too: torch may hand memory that it allocates here to the current stream's work
before the other stream is done with it.

Forward only: nothing here has a gradient.  Inputs that require one are taken as
they are, and what is computed from them is cut off from them, as by ``detach``.
"""

from __future__ import annotations

from functools import lru_cache

from .spconv import (_ACTS, _SCORES, BF16, F16, F32, FP8, _check, load_library, spconv_experts_fp8_workspace,
                     spconv_linear, spconv_linear_fp8_workspace)

BLOCK = 128
# bound by _bind, at the first call that needs torch: a call's host time is that of its launch
# (3.5 us) and what stands here, so nothing is looked up twice
_torch = None
_TYPES = {}
_lib = _device = _raw_stream = None
# sizes are asked for on every call
_linear_workspace = lru_cache(maxsize=1024)(spconv_linear_fp8_workspace)
_experts_workspace = lru_cache(maxsize=1024)(spconv_experts_fp8_workspace)


def _bind():
    global _torch, _lib, _device, _raw_stream
    import torch
    _lib = load_library()
    # what torch.cuda.current_device asks once the GPU is in use, as it is where a tensor lies there
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if _raw_stream is None:
        def _raw_stream(device):
            return torch.cuda.current_stream(device).cuda_stream
    _TYPES.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
    _torch = torch


def _type(dtype, what: str) -> int:
    """The library's number for a torch element type."""
    if _torch is None:
        _bind()
    try:
        return _TYPES[dtype]
    except KeyError:
        raise ValueError("%s must be float32, float16 or bfloat16, not %s" % (what, dtype)) from None


def _matrix(x, what: str):
    """(rows, cols, row stride, device) of a matrix on the current GPU whose rows are contiguous."""
    device = x.get_device()
    if device < 0 or x.dim() != 2 or device != _device():
        raise ValueError("%s must be a matrix on the current GPU" % what)
    rows, cols = x.shape
    ld, step = x.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s must have contiguous rows" % what)
    return rows, cols, ld if rows > 1 else cols, device


def _handle(stream, device) -> int:
    """The address of a torch stream, or of torch's current one on the device."""
    if stream is None:
        return _raw_stream(device)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _gpu_of(t, what: str):
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % what)
    return t.device


def _given(t, shape, dtype, device, what: str):
    """t, checked to be a contiguous tensor of this shape and type on this device."""
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s" % (what, dtype, shape, device))
    return t


def _bytes(workspace, device) -> int:
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on %s" % device)
    return workspace.numel() * workspace.element_size()


def _blocks(n: int) -> int:
    return -(-n // BLOCK)


def quantize_fp8(x, block_rows: int = 1, q=None, scale=None, stream=None):
    """A matrix [rows, cols] as 8-bit codes [rows, 128 kb] (float8_e4m3fn, kb =
    ceil(cols / 128)) and scales: [kb, rows] with block_rows = 1 (activations),
    [ceil(rows / 128), kb] with block_rows = 128 (weights)."""
    kind = _type(x.dtype, "x")
    rows, cols, ld, device = _matrix(x, "x")
    if block_rows not in (1, BLOCK):
        raise ValueError("block_rows must be 1 or %d" % BLOCK)
    kb = -(-cols // BLOCK)
    shape = (kb, rows) if block_rows == 1 else (-(-rows // BLOCK), kb)
    if q is None:
        q = x.new_empty((rows, kb * BLOCK), dtype=_torch.float8_e4m3fn)
    else:
        _given(q, (rows, kb * BLOCK), _torch.float8_e4m3fn, x.device, "q")
    if scale is None:
        scale = x.new_empty(shape, dtype=_torch.float32)
    else:
        _given(scale, shape, _torch.float32, x.device, "scale")
    if rows and cols:
        _check(_lib.spconv_quantize_fp8(x.data_ptr(), kind, ld, rows, cols, block_rows, q.data_ptr(), scale.data_ptr(),
                                        _handle(stream, device)))
    return q, scale


class Fp8Linear:
    """A dense layer y = act(x W^T + b) with W [cout, cin] in 8 bits:
    ``quantize_fp8(W, 128)``'s codes and scales.  It keeps the tensors given."""

    def __init__(self, w, w_scale, cout: int, cin: int, bias=None, act: str = "none"):
        import torch
        if act not in ("none", "relu", "relu6"):
            raise ValueError("act must be 'none', 'relu' or 'relu6'")
        kb, dev = _blocks(cin), _gpu_of(w, "w")
        self.w = _given(w, (cout, kb * BLOCK), torch.float8_e4m3fn, dev, "w")
        self.w_scale = _given(w_scale, (_blocks(cout), kb), torch.float32, dev, "w_scale")
        self.bias = None if bias is None else _given(bias, (cout,), torch.float32, dev, "bias")
        self.cout, self.cin, self.act, self.device = int(cout), int(cin), act, dev

    @classmethod
    def from_dense(cls, weight, bias=None, act: str = "none"):
        """The layer of a weight [cout, cin] in float32, float16 or bfloat16."""
        w, scale = quantize_fp8(weight, BLOCK)
        return cls(w, scale, weight.shape[0], weight.shape[1], bias, act)

    def workspace_bytes(self, n: int, dtype) -> int:
        """Workspace of run() for n rows of a torch dtype that is not quantised yet."""
        return _linear_workspace(_type(dtype, "x"), n, self.cin, self.cout)

    def run(self, x, x_scale=None, y=None, dtype=None, workspace=None, stream=None):
        """y [n, cout] for x [n, cin], or for quantize_fp8's codes and scales
        (then ``dtype`` or ``y`` gives y's type; it is x's otherwise)."""
        if x_scale is None:
            kind = _type(x.dtype, "x")
            n, cols, ld, device = _matrix(x, "x")
            if cols != self.cin or device != self.device.index:
                raise ValueError("x must have %d channels and be on %s" % (self.cin, self.device))
            dtype = dtype or (x.dtype if y is None else y.dtype)
        else:
            n, kind, ld, device = int(x.shape[0]), FP8, 0, self.device.index
            if _torch is None:
                _bind()
            if device != _device():
                raise ValueError("the layer must be on the current GPU")
            _given(x, (n, _blocks(self.cin) * BLOCK), _torch.float8_e4m3fn, self.device, "x")
            _given(x_scale, (_blocks(self.cin), n), _torch.float32, self.device, "x_scale")
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
                workspace = x.new_empty(size, dtype=_torch.uint8)
            else:
                size = _bytes(workspace, self.device)
            space = workspace.data_ptr()
        if n:
            _check(_lib.spconv_linear_fp8(
                x.data_ptr(), kind, ld, None if x_scale is None else x_scale.data_ptr(), self.w.data_ptr(),
                self.w_scale.data_ptr(), None if self.bias is None else self.bias.data_ptr(), _ACTS[self.act],
                y.data_ptr(), _type(dtype, "y"), n, self.cin, self.cout, space, size, _handle(stream, device)))
        return y


def route(logits, k: int, score: str = "softmax", bias=None, groups: int = 1, groups_kept: int = 1,
          group_top: int = 1, renorm: bool = True, factor: float = 1.0, ids=None, weights=None, stream=None):
    """The k experts (int32) of each token and their weights (float32), both
    [n, k], from a router's logits [n, experts]; spconv_route in
    include/spconv.h defines them."""
    kind = _type(logits.dtype, "logits")
    n, experts, ld, device = _matrix(logits, "logits")
    if score not in _SCORES:
        raise ValueError("score must be 'softmax' or 'sigmoid'")
    if bias is not None:
        _given(bias, (experts,), _torch.float32, logits.device, "bias")
    if ids is None:
        ids = logits.new_empty((n, max(k, 0)), dtype=_torch.int32)
    else:
        _given(ids, (n, k), _torch.int32, logits.device, "ids")
    if weights is None:
        weights = logits.new_empty((n, max(k, 0)), dtype=_torch.float32)
    else:
        _given(weights, (n, k), _torch.float32, logits.device, "weights")
    _check(_lib.spconv_route(logits.data_ptr(), kind, ld, None if bias is None else bias.data_ptr(), _SCORES[score], n,
                             experts, groups, groups_kept, group_top, k, renorm, factor, ids.data_ptr(),
                             weights.data_ptr(), _handle(stream, device)))
    return ids, weights


class Experts:
    """The gated feed-forward networks of a layer's experts, in 8 bits: codes
    and scales of W1 and W3 [experts, 2, inner, hidden] and of W2 [experts,
    hidden, inner], each matrix quantised by 128 x 128 blocks of its own.  It
    keeps the tensors given."""

    def __init__(self, w13, w13_scale, w2, w2_scale, hidden: int, inner: int):
        import torch
        f8, f32, dev = torch.float8_e4m3fn, torch.float32, _gpu_of(w13, "w13")
        hb, ib, e = _blocks(hidden), _blocks(inner), int(w13.shape[0])
        self.w13 = _given(w13, (e, 2, inner, hb * BLOCK), f8, dev, "w13")
        self.w13_scale = _given(w13_scale, (e, 2, ib, hb), f32, dev, "w13_scale")
        self.w2 = _given(w2, (e, hidden, ib * BLOCK), f8, dev, "w2")
        self.w2_scale = _given(w2_scale, (e, hb, ib), f32, dev, "w2_scale")
        self.experts, self.hidden, self.inner, self.device = e, int(hidden), int(inner), dev

    @classmethod
    def from_dense(cls, w1, w3, w2):
        """The experts of W1 and W3 [experts, inner, hidden] and W2 [experts,
        hidden, inner] in float32, float16 or bfloat16."""
        import torch
        e, inner, hidden = w1.shape
        hb, ib = _blocks(hidden), _blocks(inner)
        f8, f32, dev = torch.float8_e4m3fn, torch.float32, w1.device
        w13 = torch.empty((e, 2, inner, hb * BLOCK), dtype=f8, device=dev)
        w13_scale = torch.empty((e, 2, ib, hb), dtype=f32, device=dev)
        q2 = torch.empty((e, hidden, ib * BLOCK), dtype=f8, device=dev)
        q2_scale = torch.empty((e, hb, ib), dtype=f32, device=dev)
        for i in range(e):
            quantize_fp8(w1[i], BLOCK, w13[i, 0], w13_scale[i, 0])
            quantize_fp8(w3[i], BLOCK, w13[i, 1], w13_scale[i, 1])
            quantize_fp8(w2[i], BLOCK, q2[i], q2_scale[i])
        return cls(w13, w13_scale, q2, q2_scale, hidden, inner)

    def workspace_bytes(self, n: int, k: int) -> int:
        """Workspace of run() for n tokens of k experts."""
        return _experts_workspace(n, k, self.experts, self.hidden, self.inner)

    def run(self, x, ids, weights, y=None, workspace=None, stream=None):
        """y [n, hidden] = the sum of the experts' outputs for x [n, hidden],
        with ids (int32) and weights (float32) [n, k] as route() gives them."""
        kind = _type(x.dtype, "x")
        n, cols, ld, device = _matrix(x, "x")
        if cols != self.hidden or device != self.device.index:
            raise ValueError("x must have %d channels and be on %s" % (self.hidden, self.device))
        if ids.dim() != 2:
            raise ValueError("ids must be a matrix [n, k]")
        k = ids.shape[1]
        _given(ids, (n, k), _torch.int32, self.device, "ids")
        _given(weights, (n, k), _torch.float32, self.device, "weights")
        if y is None:
            y = x.new_empty((n, cols))
        else:
            _given(y, (n, cols), x.dtype, self.device, "y")
        if workspace is None:
            size = self.workspace_bytes(n, k)
            workspace = x.new_empty(size, dtype=_torch.uint8)
        else:
            size = _bytes(workspace, self.device)
        _check(_lib.spconv_experts_fp8(
            x.data_ptr(), kind, ld, ids.data_ptr(), weights.data_ptr(), self.w13.data_ptr(), self.w13_scale.data_ptr(),
            self.w2.data_ptr(), self.w2_scale.data_ptr(), y.data_ptr(), n, k, self.experts, self.hidden, self.inner,
            workspace.data_ptr(), size, _handle(stream, device)))
        return y


class ExpertLayer:
    """A mixture-of-experts layer for one batch size, as a model's forward pass
    runs it: the router's logits (``spconv_linear``, fp32), ``route``, the chosen
    ``Experts``, the residual sum and, where ``head`` is given, a dense layer in
    8 or 4 bits (``Fp8Linear``, ``Mxfp4Linear``) on top.

    ``router`` is the router's weight [experts, hidden] in float32; ``score``,
    ``bias``, ``groups``, ... are route()'s.  ``norm`` and ``head_norm`` are gains
    [hidden]: with the one the router and the experts read rms_norm(x) with
    ``eps`` (the residual stays x), with the other the head reads the sum's, which
    an ``Fp8Linear`` takes as the norm's own codes.  ``sampler``, a dict of
    sample()'s temperature, top_k, top_p and min_p, ends the step with the
    choice of ``tokens`` [batch] from the output as logits and the random numbers
    in ``u`` [batch].  Buffers are made once; every step is queued on torch's
    current stream.  ``capture`` records the steps into one graph
    (torch.cuda.CUDAGraph over HIP graphs) and ``replay`` launches it on what
    ``x`` and ``u`` hold.
    """

    def __init__(self, router, experts: Experts, k: int, batch: int, dtype=None, head=None,
                 residual: bool = True, score: str = "softmax", bias=None, groups: int = 1, groups_kept: int = 1,
                 group_top: int = 1, renorm: bool = True, factor: float = 1.0, norm=None, head_norm=None,
                 eps: float = 1e-6, sampler: dict = None):
        import torch

        from . import serving
        dev, f32 = experts.w13.device, torch.float32
        dtype = dtype or torch.bfloat16
        _type(dtype, "dtype")
        self.router = _given(router, (experts.experts, experts.hidden), f32, dev, "router")
        if head is not None and head.cin != experts.hidden:
            raise ValueError("head must take %d channels" % experts.hidden)
        if head is None and head_norm is not None:
            raise ValueError("head_norm needs a head")
        for gain, what in ((norm, "norm"), (head_norm, "head_norm")):
            if gain is not None:
                _given(gain, (experts.hidden,), f32 if gain.dtype != dtype else dtype, dev, what)
        self.serving, self.norm, self.head_norm, self.eps, self.sampler = serving, norm, head_norm, float(eps), sampler
        self.experts, self.head, self.k, self.residual = experts, head, int(k), residual
        self.choice = dict(score=score, bias=bias, groups=groups, groups_kept=groups_kept, group_top=group_top,
                           renorm=renorm, factor=factor)

        def make(cols, kind):
            return torch.zeros((batch, cols), dtype=kind, device=dev)

        self.x = make(experts.hidden, dtype)  # the static input
        self.x32 = make(experts.hidden, f32)
        self.logits = make(experts.experts, f32)
        self.ids, self.weights = make(k, torch.int32), make(k, f32)
        self.y = make(experts.hidden, dtype)
        self.out = self.y if head is None else make(head.cout, dtype)
        self.space = torch.empty(experts.workspace_bytes(batch, k), dtype=torch.uint8, device=dev)
        self.head_space = None if head is None else torch.empty(head.workspace_bytes(batch, dtype), dtype=torch.uint8,
                                                                device=dev)
        self.h = self.x if norm is None else make(experts.hidden, dtype)
        # the head's input: rows, or with a norm before an 8-bit head its codes and scales
        self.top = self.y if head_norm is None else None if isinstance(head, Fp8Linear) else make(experts.hidden, dtype)
        if self.top is None and head is not None:
            kb = _blocks(experts.hidden)
            self.q = torch.zeros((batch, kb * BLOCK), dtype=torch.float8_e4m3fn, device=dev)
            self.q_scale = torch.zeros((kb, batch), dtype=f32, device=dev)
        if sampler is not None:
            self.u, self.tokens = torch.zeros(batch, dtype=f32, device=dev), torch.zeros(batch, dtype=torch.int32, device=dev)
            self.sample_space = torch.empty(
                max(serving.spconv_sample_workspace(_type(dtype, "dtype"), batch, self.out.shape[1]), 1),
                dtype=torch.uint8, device=dev)
        self.graph = None

    def forward(self, x=None):
        """Queue the layer (copying x into the static input first when given); returns the output buffer."""
        if x is not None:
            self.x.copy_(x)
        e = self.experts
        if self.norm is None:
            self.x32.copy_(self.x)
        else:
            self.serving.rms_norm(self.x, self.norm, self.eps, y=self.x32)
            self.h.copy_(self.x32)
        spconv_linear(self.x32, self.router, None, "none", self.logits, self.x.shape[0], e.hidden, e.experts)
        route(self.logits, self.k, ids=self.ids, weights=self.weights, **self.choice)
        e.run(self.h, self.ids, self.weights, self.y, self.space)
        if self.head_norm is not None:
            self._normed_head()
        else:
            if self.residual:
                self.y.add_(self.x)
            if self.head is not None:
                self.head.run(self.y, y=self.out, workspace=self.head_space)
        if self.sampler is not None:
            self.serving.sample(self.out, self.u, ids=self.tokens, workspace=self.sample_space, **self.sampler)
        return self.out

    def _normed_head(self):
        """The residual sum (into y), its norm and the head: the sum and the norm are one pass over the rows."""
        x, total = (self.x, self.y) if self.residual else (self.y, None)
        if self.top is None:
            self.serving.rms_norm_fp8(x, self.head_norm, self.eps, total, q=self.q, scale=self.q_scale, total=total)
            self.head.run(self.q, self.q_scale, y=self.out, workspace=self.head_space)
        else:
            self.serving.rms_norm(x, self.head_norm, self.eps, total, y=self.top, total=total)
            self.head.run(self.top, y=self.out, workspace=self.head_space)

    def capture(self):
        """Record the steps into one graph (after one warm-up pass)."""
        import torch
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.forward()
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.forward()
        return self.graph

    def replay(self):
        if self.graph is None:
            raise RuntimeError("capture() first")
        self.graph.replay()
        return self.out
