"""64-bit references of the 8-bit form, of products with it, of routing and of experts."""

import numpy as np

BLOCK, TOP, TINY = 128, 448.0, 2.0 ** -100
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # unit roundoff (bf16: 2^-9 rounded up)
SMALLEST = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}


def torch_dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def blocks(n):
    return -(-n // BLOCK)


def e4m3(v):
    """Rounded to the nearest e4m3 value, ties to even (|v| below 464)."""
    v = np.asarray(v, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.floor(np.log2(np.abs(v)))
    e = np.where(np.isfinite(e), np.maximum(e, -6), -6)
    step = 2.0 ** (e - 3)
    return np.round(v / step) * step


def quantize_ref(x, block_rows):
    """(code values [rows, 128 kb], scales) of a float32 matrix: every step
    rounded to 32 bits, as the form is defined."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    kb, rb = blocks(cols), -(-rows // block_rows)
    p = np.zeros((rb * block_rows, kb * BLOCK), np.float32)
    p[:rows, :cols] = x
    p = p.reshape(rb, block_rows, kb, BLOCK)
    with np.errstate(invalid="ignore", over="ignore"):
        most = np.maximum(np.abs(p).max(axis=(1, 3)), np.float32(TINY))
        scale = (most / np.float32(TOP)).astype(np.float32)
        inv = (np.float32(TOP) / most).astype(np.float32)
        q = e4m3(p * inv[:, None, :, None])
    q = q.reshape(rb * block_rows, kb * BLOCK)[:rows]
    return q, np.ascontiguousarray(scale.T) if block_rows == 1 else scale


def row_values(q, scale, cols):
    """What codes [rows, 128 kb] and scales [kb, rows] stand for, in 64 bits."""
    s = np.repeat(np.asarray(scale, np.float64).T, BLOCK, axis=1)
    return (np.asarray(q, np.float64) * s)[:, :cols]


def block_values(q, scale, cols):
    s = np.repeat(np.repeat(np.asarray(scale, np.float64), BLOCK, axis=0)[:q.shape[0]], BLOCK, axis=1)
    return (np.asarray(q, np.float64) * s)[:, :cols]


def act_ref(y, act):
    return y if act == "none" else np.clip(y, 0.0, 6.0 if act == "relu6" else np.inf)


def linear_ref(xv, wv, bias, act):
    """(y, sum of |terms|) in 64 bits."""
    b = 0.0 if bias is None else np.asarray(bias, np.float64)
    return act_ref(xv @ wv.T + b, act), np.abs(xv) @ np.abs(wv).T + np.abs(b)


def linear_tol(y, terms, cin, dtype):
    """Sums of 128 products in the matrix cores, then over blocks, each step
    at most 2^-23 of the terms' sum off (one bit more than a rounded addition,
    for additions that cut off); then one rounding to the type."""
    return terms * (BLOCK + blocks(cin) + 8) * 2.0 ** -23 + np.abs(y) * ROUND[dtype] + SMALLEST[dtype]


def code_values(q):
    """A float8 tensor's values."""
    return q.float().cpu().double().numpy()


def route_ref(logits, k, score="softmax", bias=None, groups=1, groups_kept=1, group_top=1, renorm=True, factor=1.0):
    """(ids, weights) of every token, one token and one expert after the other."""
    logits = np.minimum(np.asarray(logits, np.float64), 3.402823466e38)
    n, experts = logits.shape
    bias = np.zeros(experts) if bias is None else np.asarray(bias, np.float64)
    each = experts // groups
    ids, weights = np.full((n, k), -1, np.int32), np.zeros((n, k))
    for t in range(n):
        on = [e for e in range(experts) if logits[t, e] > -np.inf]
        s = {}
        if score == "softmax":
            top = max((logits[t, e] for e in on), default=0.0)
            total = sum(np.exp(logits[t, e] - top) for e in on)
            s = {e: np.exp(logits[t, e] - top) / total for e in on}
        else:
            with np.errstate(over="ignore"):
                s = {e: 1.0 / (1.0 + np.exp(-logits[t, e])) for e in on}
        value = {e: s[e] + bias[e] for e in on if s[e] + bias[e] > -np.inf}
        ranks = []
        for g in range(groups):
            best = sorted((v for e, v in value.items() if e // each == g), reverse=True)[:group_top]
            ranks.append((-sum(best) if best else np.inf, g))
        kept = [g for _, g in sorted(ranks)[:groups_kept]]
        chosen = sorted((e for e in value if e // each in kept), key=lambda e: (-value[e], e))[:k]
        w = np.array([s[e] for e in chosen])
        if renorm and len(w):
            w = w / w.sum() if w.sum() > 0 else np.zeros(len(w))
        ids[t, :len(chosen)] = chosen
        weights[t, :len(chosen)] = w * np.float64(np.float32(factor))
    return ids, weights


def cut_bound(xv, wv):
    """What the 8-bit instruction may lose of each product: it cuts every term
    off at 2^-17 of the largest of its block (measured: 2^-18.1), 128 terms a block."""
    out = np.zeros((xv.shape[0], wv.shape[0]))
    for b in range(0, xv.shape[1], BLOCK):
        x, w = np.abs(xv[:, b:b + BLOCK]), np.abs(wv[:, b:b + BLOCK])
        for i in range(x.shape[0]):
            out[i] += (x[i] * w).max(axis=1) * BLOCK * 2.0 ** -17
    return out


def quantize_interval(h, dh):
    """(values of h's codes, how far those of any h' with |h' - h| <= dh may
    be from them), in 64 bits: rounding is monotone, so an interval's ends bound it."""
    rows, cols = h.shape
    out, off = np.zeros_like(h), np.zeros_like(h)
    for b in range(0, cols, BLOCK):
        v, d = h[:, b:b + BLOCK], dh[:, b:b + BLOCK]
        a = np.maximum(np.abs(v).max(axis=1, keepdims=True), TINY)
        r = d.max(axis=1, keepdims=True) / a + 2.0 ** -22
        u, du = v / a * TOP, d / a * TOP
        span = du + np.abs(u) * r * 1.01
        q = e4m3(np.clip(u, -TOP, TOP))
        hi, lo = e4m3(np.clip(u + span, -TOP, TOP)), e4m3(np.clip(u - span, -TOP, TOP))
        s = a / TOP
        out[:, b:b + BLOCK] = q * s
        off[:, b:b + BLOCK] = np.maximum(hi - q, q - lo) * s * (1 + 1.01 * r) + np.abs(q) * s * r * 1.01
    return out, off


def experts_ref(x, ids, weights, layer, cut=False):
    """(y, tolerance before the last rounding) in 64 bits; `cut`: with the 8-bit instruction's loss."""
    n, k = ids.shape
    xq, xs = quantize_ref(x, 1)
    xv = row_values(xq, xs, layer.hidden)
    y, tol = np.zeros((n, layer.hidden)), np.zeros((n, layer.hidden))
    w13, s13 = code_values(layer.w13), layer.w13_scale.cpu().numpy()
    w2, s2 = code_values(layer.w2), layer.w2_scale.cpu().numpy()
    for e in range(layer.experts):
        token, slot = np.nonzero(ids == e)
        if len(token) == 0:
            continue
        xe = xv[token]
        (g, dg), (u, du) = ((lambda w: (xe @ w.T, np.abs(xe) @ np.abs(w).T * (BLOCK + blocks(layer.hidden)) * 2.0 ** -23 +
                                        (cut_bound(xe, w) if cut else 0)))(block_values(w13[e, i], s13[e, i], layer.hidden))
                            for i in (0, 1))
        with np.errstate(over="ignore"):
            silu = g / (1 + np.exp(-g))
        # |silu'| <= 1.1; the gate's own arithmetic: 16 last places
        dh = 1.1 * dg * (np.abs(u) + du) + np.abs(silu) * du + np.abs(silu * u) * 2.0 ** -20
        hv, dv = quantize_interval(silu * u, dh)
        w = block_values(w2[e], s2[e], layer.inner)
        z = hv @ w.T
        dz = (dv @ np.abs(w).T + (np.abs(hv) + dv) @ np.abs(w).T * (BLOCK + blocks(layer.inner)) * 2.0 ** -23 +
              (cut_bound(hv, w) if cut else 0))
        p = weights[token, slot].astype(np.float64)[:, None]
        np.add.at(y, token, z * p)
        np.add.at(tol, token, (dz + np.abs(z) * (k + 4) * 2.0 ** -23) * np.abs(p))
    return y, tol
