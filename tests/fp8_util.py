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
