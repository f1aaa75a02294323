"""Operators around the dense layers of a language model that is served, as
cases that can be timed.

Four kinds of case:

* ``norm``: the root-mean-square norm of a row, with the residual's addition
  in front, as rows of the input's type or as 8-bit codes with a scale for
  each 128 channels;
* ``quantize``: a matrix to 4-bit floating point (e2m1) with a power of two for
  each 32 columns of a row;
* ``linear``: y = act(q(x) W^T + b) with W in that form and x quantised on
  the way;
* ``sample``: the next token of each sequence from its logits and a given
  random number, by temperature, top-k, top-p and min-p.

Inputs follow from the seed alone: activations ~ N(0, 1) with a few channels
10 times as large (as after a residual stream), weights ~ N(0, 1 / cin), a
norm's gains ~ N(1, 0.04), logits ~ N(0, 4) with 20 tokens of each row ahead.
"""

import math
from types import SimpleNamespace

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
CLAMP = {"none": (None, None), "relu": (0.0, None), "relu6": (0.0, 6.0)}
EPS = 1e-6
BLOCK8 = 128  # channels of an 8-bit block
TOP8 = 448.0  # the largest e4m3 value
TINY8 = 2.0 ** -100  # the least magnitude that an 8-bit block's scale stands for
BLOCK4 = 32  # channels of a 4-bit block
LINE4 = 256  # channels of 128 bytes of 4-bit codes: rows are padded to whole lines
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # the magnitudes of e2m1
MOST_LINEAR = 8192 * 4096 * 4096
MOST_LOGITS = 256 * 50001


def _up(n, block):
    return (n + block - 1) // block


def _norm(name, rows, cols, dtype, residual=None, fp8=False):
    """residual: the type of the residual stream, or None for a norm alone."""
    return dict(name=name, kind="norm", rows=rows, cols=cols, dtype=dtype, residual=residual, fp8=fp8)


def _quantize(name, rows, cols, dtype):
    return dict(name=name, kind="quantize", rows=rows, cols=cols, dtype=dtype)


def _linear(name, n, cin, cout, dtype, act="none", bias=False):
    return dict(name=name, kind="linear", n=n, cin=cin, cout=cout, dtype=dtype, act=act, bias=bias)


def _sample(name, n, vocab, dtype, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, each=False, masked=False):
    """each: every row has parameters of its own, on the GPU, in place of these;
    masked: tokens that a grammar forbids have logits of -inf."""
    return dict(name=name, kind="sample", n=n, vocab=vocab, dtype=dtype, temperature=temperature, top_k=top_k,
                top_p=top_p, min_p=min_p, each=each, masked=masked)


def listed():
    return [
        # one token between two layers: latency
        _norm("norm_1x1280_f16_residual", 1, 1280, "f16", "f16"),
        # odd rows and channels, no residual
        _norm("norm_777x1000_f32", 777, 1000, "f32"),
        # a long prompt before an 8-bit layer: bound by traffic
        _norm("norm_8192x4096_bf16_residual_fp8", 8192, 4096, "bf16", "bf16", True),
        # a few tokens' activations, before several products
        _quantize("quantize4_16x1280_f16", 16, 1280, "f16"),
        # a layer's weight, once at load, or the activations of a long prompt
        _quantize("quantize4_8192x4096_bf16", 8192, 4096, "bf16"),
        # one token: bound by the weight's bytes
        _linear("linear4_1x4096_4096_bf16", 1, 4096, 4096, "bf16"),
        # one step of a batch of sequences over a wide layer
        _linear("linear4_24x4096_8192_bf16", 24, 4096, 8192, "bf16"),
        # odd rows, channels that leave the last block short, bias and clamp
        _linear("linear4_777x1000_2500_f16", 777, 1000, 2500, "f16", "relu6", True),
        # a long prompt: bound by the product
        _linear("linear4_8192x4096_4096_bf16", 8192, 4096, 4096, "bf16"),
        # one sequence with the usual settings: latency
        _sample("sample_1x32000_f32_k50_p95", 1, 32000, "f32", 0.8, 50, 0.95),
        # a batch of requests with settings of their own, a large vocabulary
        _sample("sample_64x131072_bf16_each", 64, 131072, "bf16", each=True),
        # a large batch drawn from all of its odd vocabulary
        _sample("sample_256x50001_f32_all", 256, 50001, "f32", 0.7),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high):
    """Mostly a multiple of 64, as in use; now and then any number."""
    v = _log(rng, low, high)
    return max(64, v // 64 * 64) if rng.random() < 0.7 else v


def draw(rng):
    """A case of the listed ranges: one row to 8192 (256 of logits), 64 to
    8192 channels, 1000 to 160000 tokens; no more work than the largest listed."""
    kind = rng.choice(("norm", "norm", "quantize", "linear", "linear", "sample", "sample"))
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    if kind == "norm":
        cols = _size(rng, 64, 8192)
        residual = rng.choice((None, dtype, dtype, "f32"))
        case = _norm(None, _log(rng, 1, min(8192, 8192 * 4096 // cols)), cols, dtype, residual, rng.random() < 0.5)
    elif kind == "quantize":
        cols = _size(rng, 64, 8192)
        case = _quantize(None, _log(rng, 1, min(8192, 8192 * 4096 // cols)), cols, dtype)
    elif kind == "linear":
        cin, cout = _size(rng, 64, 8192), _size(rng, 64, 8192)
        n = _log(rng, 1, min(8192, MOST_LINEAR // (cin * cout)))
        case = _linear(None, n, cin, cout, dtype, rng.choice(("none", "none", "relu", "relu6")), rng.random() < 0.5)
    else:
        vocab = _log(rng, 1000, 160000)
        case = _sample(None, _log(rng, 1, min(256, MOST_LOGITS // vocab)), vocab, dtype,
                       rng.choice((0.0, 0.5, 0.8, 1.0, 1.3)), rng.choice((0, 0, 1, 40, 50, 1000)),
                       rng.choice((1.0, 1.0, 0.5, 0.9, 0.95, 0.99)), rng.choice((0.0, 0.0, 0.02, 0.1)),
                       rng.random() < 0.4, rng.random() < 0.3)
    del case["name"]
    return case


def work(case):
    """Each input read once and each output written once."""
    kind = case["kind"]
    size = SIZES[case["dtype"]]
    if kind == "norm":
        rows, cols = case["rows"], case["cols"]
        values = rows * cols
        stream = 2 * SIZES[case["residual"]] * values if case["residual"] else 0
        kb = _up(cols, BLOCK8)
        out = rows * kb * (BLOCK8 + 4) if case["fp8"] else values * size
        return {"bytes": values * size + stream + out + cols * size, "flops": 6 * values}
    if kind == "quantize":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": rows * (cols * size + _up(cols, LINE4) * 136), "flops": 3 * rows * cols}
    if kind == "linear":
        n, cin, cout = case["n"], case["cin"], case["cout"]
        weight = cout * _up(cin, BLOCK4) * 17 + (4 * cout if case["bias"] else 0)
        return {"bytes": weight + size * n * (cin + cout), "flops": 2 * n * cin * cout}
    n, vocab = case["n"], case["vocab"]
    return {"bytes": n * (vocab * size + (24 if case["each"] else 8)), "flops": 4 * n * vocab}


# ---- inputs ----

def _activations(n, c, dtype, gen):
    x = torch.randn((n, c), generator=gen, device=DEVICE)
    loud = torch.randint(0, c, (max(1, c // 100),), generator=gen, device=DEVICE)
    x[:, loud] *= 10
    return x.to(DTYPES[dtype])


def _logits(case, gen):
    n, vocab = case["n"], case["vocab"]
    logits = torch.randn((n, vocab), generator=gen, device=DEVICE) * 2
    ahead = torch.randint(0, vocab, (n, 20), generator=gen, device=DEVICE)
    logits.scatter_add_(1, ahead, torch.rand((n, 20), generator=gen, device=DEVICE) * 10)
    if case["masked"]:
        logits[torch.rand((n, vocab), generator=gen, device=DEVICE) < 0.5] = -math.inf
    return logits.to(DTYPES[case["dtype"]])


def _pick(values, n, gen):
    return torch.tensor(values, device=DEVICE)[torch.randint(0, len(values), (n,), generator=gen, device=DEVICE)]


def _parts(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    kind = case["kind"]
    s = SimpleNamespace(case=case)
    if kind == "norm":
        s.x = _activations(case["rows"], case["cols"], case["dtype"], gen)
        s.residual = _activations(case["rows"], case["cols"], case["residual"], gen) if case["residual"] else None
        s.gain = (1 + 0.2 * torch.randn(case["cols"], generator=gen, device=DEVICE)).to(DTYPES[case["dtype"]])
    elif kind == "quantize":
        s.x = _activations(case["rows"], case["cols"], case["dtype"], gen)
    elif kind == "linear":
        s.x = _activations(case["n"], case["cin"], case["dtype"], gen)
        w = torch.randn((case["cout"], case["cin"]), generator=gen, device=DEVICE) / math.sqrt(case["cin"])
        s.w, s.w_scale = _to_blocks4(w)
        s.bias = torch.randn(case["cout"], generator=gen, device=DEVICE) if case["bias"] else None
    else:
        n = case["n"]
        s.logits = _logits(case, gen)
        s.u = torch.rand(n, generator=gen, device=DEVICE)
        if case["each"]:
            s.temperature = _pick((0.0, 0.3, 0.7, 1.0, 1.0, 1.5), n, gen)
            s.top_k = _pick((0, 0, 1, 20, 50, 500), n, gen).int()
            s.top_p = _pick((1.0, 1.0, 0.5, 0.9, 0.95, 0.99), n, gen)
            s.min_p = _pick((0.0, 0.0, 0.0, 0.02, 0.1), n, gen)
        else:
            s.temperature, s.top_k, s.top_p, s.min_p = (case[p] for p in ("temperature", "top_k", "top_p", "min_p"))
    return s


def prepare(case, seed):
    s = _parts(case, seed)
    if own and case["kind"] == "linear":
        # the handle that a program keeps for a layer: it holds the weight as it is
        import paper_1911_09723_amd as amd
        s.layer = amd.Mxfp4Linear(s.w, s.w_scale, case["cout"], case["cin"], s.bias, case["act"])
    return s


def run(state):
    """The quantiser's codes, two a byte, and its powers of two are whole
    numbers: they are compared bit for bit."""
    case, kind = state.case, state.case["kind"]
    if own:
        if kind == "linear":
            return state.layer.run(state.x)
        import paper_1911_09723_amd as amd
        if kind == "norm":
            norm = amd.rms_norm_fp8 if case["fp8"] else amd.rms_norm
            return norm(state.x, state.gain, EPS, state.residual)
        if kind == "quantize":
            return amd.quantize_mxfp4(state.x)
        return amd.sample(state.logits, state.u, state.temperature, state.top_k, state.top_p, state.min_p)
    if kind == "norm":
        return _norm_plain(state)
    if kind == "quantize":
        return _to_blocks4(state.x)
    if kind == "linear":
        x, w = _values4(*_to_blocks4(state.x), case["cin"]), _values4(state.w, state.w_scale, case["cin"])
        y = x @ w.T
        if state.bias is not None:
            y = y + state.bias
        return _act(y, case["act"]).to(state.x.dtype)
    return _sample_plain(state)


# ---- the plain forms ----

def _padded(x, cols):
    if x.shape[1] == cols:
        return x
    p = torch.zeros((x.shape[0], cols), dtype=x.dtype, device=x.device)
    p[:, :x.shape[1]] = x
    return p


def _norm_plain(s):
    h = s.x.float() if s.residual is None else s.x.float() + s.residual.float()
    y = h * (1 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + EPS)) * s.gain.float()
    out = _to_blocks8(y) if s.case["fp8"] else (y.to(s.x.dtype),)
    if s.residual is not None:
        out = out + (h.to(s.residual.dtype),)
    return out if len(out) > 1 else out[0]


def _to_blocks8(y):
    """8-bit codes [rows, 128 kb] and scales [kb, rows]."""
    rows, kb = y.shape[0], _up(y.shape[1], BLOCK8)
    v = _padded(y, kb * BLOCK8).view(rows, kb, BLOCK8)
    most = v.abs().amax(dim=2).clamp_min(TINY8)
    top = torch.full_like(most, TOP8)
    q = (v * (top / most)[..., None]).clamp_(-TOP8, TOP8).view(rows, -1).to(torch.float8_e4m3fn)
    return q, (most / top).T.contiguous()


def _to_blocks4(x):
    """4-bit codes, two a byte (the even column in the lower half), [rows, 128
    lines], and the exponents of their powers of two, off by 127, [lines, rows, 8]."""
    rows, lines = x.shape[0], _up(x.shape[1], LINE4)
    v = _padded(x.float(), lines * LINE4).view(rows, lines, 8, BLOCK4)
    bits = v.abs().amax(dim=3).view(torch.int32)
    lost = bits >= 0x7f800000  # an infinity or a NaN
    # the least power of two whose quotients stay below 7, which rounds to 6
    power = (((bits + 0x200000) >> 23) - 2).clamp_min(0)
    inverse = torch.where(power < 254, (254 - power) << 23, 1 << 22).view(torch.float32)
    v = torch.where(lost[..., None], 0.0, v * inverse[..., None])
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    code = torch.round(a / step) + torch.where(a < 2, 0.0, torch.where(a < 4, 2.0, 4.0))  # halfway goes to the even code
    code = (code + 8 * torch.signbit(v)).to(torch.uint8)
    code = code.view(rows, -1, 2)
    scale = torch.where(lost, 255, power).to(torch.uint8)
    return code[..., 0] | code[..., 1] << 4, scale.transpose(0, 1).contiguous()


def _values4(q, scale, cols):
    """What 4-bit codes and their powers of two stand for."""
    rows = q.shape[0]
    codes = torch.stack((q & 15, q >> 4), dim=2).view(rows, -1, BLOCK4).long()
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=q.device)[codes]
    power = scale.transpose(0, 1).reshape(rows, -1).int()
    power = torch.where(power > 0, power << 23, 1 << 22).view(torch.float32)
    power = torch.where(power < math.inf, power, math.nan)
    return (level * power[..., None]).view(rows, -1)[:, :cols]


def _act(y, act):
    low, high = CLAMP[act]
    return y if low is None else y.clamp_(min=low, max=high)


def _sample_plain(s):
    """In 64 bits: the choice hangs on sums next to a border."""
    logits = s.logits.double()
    n, vocab = logits.shape
    logits = torch.where(logits > -math.inf, logits.clamp(max=torch.finfo(torch.float32).max), -math.inf)
    columns = (torch.as_tensor(p, device=logits.device).expand(n)[:, None]
               for p in (s.temperature, s.top_k, s.top_p, s.min_p))
    temperature, top_k, top_p, min_p = columns
    temperature, top_p, min_p = (p.float().double() for p in (temperature, top_p, min_p))
    value, order = logits.sort(dim=1, descending=True, stable=True)
    on = value > -math.inf
    none = ~on[:, :1]
    first = torch.where(none, 0.0, value[:, :1])
    place = torch.arange(vocab, device=logits.device)
    greedy = temperature <= 0
    weight = torch.where(on, torch.exp((value - first) / torch.where(greedy, 1.0, temperature)), 0.0)
    weight = torch.where((place < torch.where(top_k > 0, top_k, vocab)), weight, 0.0)
    before = weight.cumsum(dim=1) - weight
    kept = (before < top_p * weight.sum(dim=1, keepdim=True)) | (top_p >= 1)
    kept = torch.where(greedy, False, kept & (weight >= min_p)) | (place == 0)
    weight = torch.where(kept, weight, 0.0)
    weight = torch.zeros_like(weight).scatter_(1, order, weight)  # back in the order of the tokens
    running = weight.cumsum(dim=1)
    past = running > s.u.double()[:, None] * running[:, -1:]
    ids = torch.where(past, place, vocab).amin(dim=1)
    return torch.where(none[:, 0], -1, ids).int()


# ---- the same from the definition, in 64 bits ----

def _nearest(v, levels):
    """The index of the level nearest to each v >= 0; halfway the even index."""
    best, found = torch.full_like(v, math.inf), torch.zeros_like(v, dtype=torch.int64)
    for i, level in enumerate(levels):
        off = (v - level).abs()
        nearer = (off < best) | ((off == best) & (i % 2 == 0))
        best, found = torch.where(nearer, off, best), torch.where(nearer, i, found)
    return found


def _e4m3(v):
    """v rounded to the nearest multiple of its e4m3 step, ties to even."""
    exponent = torch.frexp(v).exponent.clamp(min=-5) - 1  # 2^-6 is the least normal value
    step = torch.ldexp(torch.ones_like(v), exponent - 3)
    return torch.round(v / step) * step


def _exact_norm(s):
    h = s.x.double()
    if s.residual is not None:
        h = h + s.residual.double()
    y = h / torch.sqrt(h.pow(2).sum(dim=1, keepdim=True) / h.shape[1] + EPS) * s.gain.double()
    out = [y]
    if s.case["fp8"]:
        rows, cols = y.shape
        kb = _up(cols, BLOCK8)
        q = torch.zeros((rows, kb * BLOCK8), dtype=torch.float64, device=y.device)
        scale = torch.zeros((kb, rows), dtype=torch.float64, device=y.device)
        for b in range(kb):
            part = y[:, b * BLOCK8:(b + 1) * BLOCK8]
            most = part.abs().max(dim=1).values.clamp(min=TINY8)
            scale[b] = most / TOP8
            q[:, b * BLOCK8:b * BLOCK8 + part.shape[1]] = _e4m3(part / most[:, None] * TOP8)
        out = [q, scale]
    if s.residual is not None:
        out.append(h)
    return tuple(out) if len(out) > 1 else out[0]


def _exact_blocks4(x):
    """Codes (0 to 15) [rows, 256 lines] and exponents [rows, 8 lines] of finite rows."""
    rows, cols = x.shape
    lines = _up(cols, LINE4)
    codes = torch.zeros((rows, lines * LINE4), dtype=torch.int64, device=x.device)
    power = torch.full((rows, lines * 8), -127, dtype=torch.int64, device=x.device)
    for b in range(_up(cols, BLOCK4)):
        part = x[:, b * BLOCK4:(b + 1) * BLOCK4].double()
        most = part.abs().max(dim=1).values
        e = torch.floor(torch.log2(most.clamp(min=2.0 ** -140))) - 2
        e = (e + (most >= 7 * torch.exp2(e))).clamp(min=-127)
        v = part / torch.exp2(e)[:, None]
        codes[:, b * BLOCK4:b * BLOCK4 + part.shape[1]] = _nearest(v.abs(), LEVELS) + 8 * torch.signbit(v)
        power[:, b] = e.long()
    return codes, power


def _exact_quantize(s):
    codes, power = _exact_blocks4(s.x)
    rows = codes.shape[0]
    q = codes[:, 0::2] + 16 * codes[:, 1::2]
    scale = torch.stack([p + 127 for p in power.split(8, dim=1)])
    return q.to(torch.uint8), scale.view(-1, rows, 8).to(torch.uint8)


def _exact_values4(codes, power, cols):
    sign = 1 - 2 * (codes >> 3).double()
    level = torch.tensor(LEVELS, dtype=torch.float64, device=codes.device).take(codes & 7)
    return (sign * level * torch.exp2(power.double()).repeat_interleave(BLOCK4, dim=1))[:, :cols]


def _exact_linear(s):
    cin, cout = s.case["cin"], s.case["cout"]
    codes = torch.zeros((cout, 2 * s.w.shape[1]), dtype=torch.int64, device=s.w.device)
    codes[:, 0::2], codes[:, 1::2] = s.w % 16, s.w // 16
    power = torch.cat([p.long() - 127 for p in s.w_scale], dim=1)
    y = _exact_values4(*_exact_blocks4(s.x), cin) @ _exact_values4(codes, power, cin).T
    return _act(y if s.bias is None else y + s.bias.double(), s.case["act"])


def _exact_sample(s):
    """Row by row; the thresholds from the sorted weights, the draw by a search."""
    n, vocab = s.logits.shape
    rows = s.logits.double().cpu()
    u = s.u.double().cpu().tolist()
    each = [p.tolist() if torch.is_tensor(p) else [torch.tensor(p).item()] * n
            for p in (s.temperature, s.top_k, s.top_p, s.min_p)]
    ids = []
    for row, r, t, k, p, least in zip(rows, u, *each):
        here = torch.nonzero(row > -math.inf)[:, 0]
        if here.numel() == 0:
            ids.append(-1)
            continue
        value, order = torch.sort(row[here], descending=True, stable=True)
        if t <= 0:
            ids.append(int(here[order[0]]))
            continue
        weight = torch.exp((value - value[0]) / t)[:k if k > 0 else vocab]
        if p < 1:
            running = torch.cumsum(weight, 0)
            weight = weight[:1 + int(torch.searchsorted(running, p * running[-1:]))]
        weight = weight[:max(1, int((weight >= least).sum()))]
        tokens, at = torch.sort(here[order[:weight.numel()]])
        running = torch.cumsum(weight[at], 0)
        ids.append(int(tokens[min(int(torch.searchsorted(running, r * running[-1:], right=True)), tokens.numel() - 1)]))
    return torch.tensor(ids, dtype=torch.int32)


def exact(case, seed):
    s = _parts(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_norm(s)
    if kind == "quantize":
        return _exact_quantize(s)
    if kind == "linear":
        return _exact_linear(s)
    return _exact_sample(s)
