"""64-bit references of norms, of the 4-bit form and its products, and of sampling."""

import math

import numpy as np

from fp8_util import ROUND, SMALLEST

LINE, BLOCK = 256, 32
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)


def lines(n):
    return -(-n // LINE)


def to_numpy(t):
    return t.detach().float().cpu().double().numpy()


# ---- norm ----

def norm_ref(x, residual=None, gain=None, eps=1e-6):
    """(y, h) in 64 bits."""
    h = x if residual is None else x + residual
    y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + np.float64(np.float32(eps)))
    return (y if gain is None else y * gain), h


def norm_tol(y, cols, dtype):
    """h is rounded once (2^-24); a thread's chain of fused steps has at most 64
    or cols / 1024 of them, 16 additions follow; the mean, eps, root and quotient are
    four roundings, the two products two more.  A relative error d of the sum is d /
    2 of the result.  Then one rounding to the type."""
    steps = max(64, cols / 1024) + 16 + 2
    return np.abs(y) * ((steps / 2 + 8) * 2.0 ** -24 * 1.01 + ROUND[dtype]) + SMALLEST[dtype]


# ---- the 4-bit form ----

def e2m1(v):
    """Codes (0 to 15) of the values nearest to v, ties to the even code."""
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    off = np.abs(a[..., None] - LEVELS)
    least = off.min(axis=-1, keepdims=True)
    near = off == least
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), near.argmax(axis=-1))
    return (code + 8 * np.signbit(v)).astype(np.uint8)


def quantize4_ref(x):
    """(codes [rows, 256 lines] of 0 to 15, scale bytes [rows, 8 lines]) of a matrix."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    n = lines(cols)
    p = np.zeros((rows, n * LINE))
    p[:, :cols] = x
    p = p.reshape(rows, n * 8, BLOCK)
    lost = ~np.isfinite(p).all(axis=2)
    p = np.where(lost[..., None], 0.0, p)
    most = np.abs(p).max(axis=2)
    _, e = np.frexp(most)  # most in [2^(e-1), 2^e)
    e = np.where(most > 0, e - 1, -2000) - 2
    e = np.maximum(e + (most >= 7 * np.ldexp(1.0, np.maximum(e, -500))), -127)
    code = e2m1(np.ldexp(p, -e[..., None]))
    code[lost] = 0
    return code.reshape(rows, -1), np.where(lost, 255, e + 127).astype(np.uint8)


def packed(code, scale):
    """The arrays as the library lays them out: codes [rows, 128 lines], scales [lines, rows, 8]."""
    rows = code.shape[0]
    q = code[:, 0::2] | code[:, 1::2] << 4
    return q, np.ascontiguousarray(scale.reshape(rows, -1, 8).transpose(1, 0, 2))


def unpacked(q, scale):
    rows = q.shape[0]
    code = np.stack([q & 15, q >> 4], axis=2).reshape(rows, -1)
    return code, scale.transpose(1, 0, 2).reshape(rows, -1)


def values4(code, scale, cols):
    """What codes and scale bytes stand for."""
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return (v.reshape(code.shape[0], -1, BLOCK) * s[..., None]).reshape(code.shape[0], -1)[:, :cols]


def linear4_tol(y, terms, cin, dtype):
    """An instruction of 128 channels adds its products and the running sum with at
    most 2^-22 of the magnitudes that it adds up (measured, 2e-7); two a line, then sums over
    at most 16 wavefronts and 16 workgroups, the bias, and one rounding to the type."""
    return terms * (2 * lines(cin) + 33) * 2.0 ** -22 + np.abs(y) * ROUND[dtype] + SMALLEST[dtype]


# ---- sampling ----

def sample_ref(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The tokens of rows of logits, each parameter a number or one for each row."""
    rows, vocab = logits.shape
    ids = []
    each = [np.broadcast_to(np.asarray(p, np.float32), rows).astype(np.float64) for p in (u, temperature, top_p, min_p)]
    ks = np.broadcast_to(np.asarray(top_k), rows)
    for l, r, t, p, least, k in zip(np.asarray(logits, np.float64), *each, ks):
        here = np.flatnonzero(l > -math.inf)
        if len(here) == 0:
            ids.append(-1)
            continue
        l = np.minimum(l, np.finfo(np.float32).max)
        order = here[np.lexsort((here, -l[here]))]
        if not t > 0:
            ids.append(order[0])
            continue
        k = vocab if k <= 0 else k
        order = order[:k]
        w = np.exp((l[order] - l[order[0]]) / t)
        if p < 1:
            run = np.cumsum(w)
            before = np.concatenate([[0.0], run[:-1]])
            order = order[:max(1, int((before < p * run[-1]).sum()))]
        least = min(max(least, 0.0), 1.0) if least == least else 0.0
        order = order[w[:len(order)] >= least]
        r = min(max(r, 0.0), 1 - 2.0 ** -24) if r == r else 0.0
        order = np.sort(order)
        run = np.cumsum(np.exp((l[order] - l[here].max()) / t))
        ids.append(order[min(int((run <= r * run[-1]).sum()), len(order) - 1)])
    return np.array(ids, np.int32)
