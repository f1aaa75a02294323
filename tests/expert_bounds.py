"""How far experts' outputs may be from 64 bits, by the type of rows and results.

The first products are exact and summed in 32 bits for every type, since their
results are rounded to codes again.  So are the second products for f32; f16 and
bf16 take the 8-bit instruction for them, and bf16 keeps their results in f16
(with a power of two for each 128) before the weighted sum.  (Token by token all
sums are 32-bit ones.)

Of one element (``bound``): 2^-23 of the terms a step, for the second products'
8-bit sums their cut (fp8_cut.cut8, with inner rows' codes at most one step of
their exponent off); f16 in between 2^-11 of a value, and 2^-25 of the power of
two below f16's normal numbers, a power that is at most 2^-14 of 448^2 * 128
times the sum of the |scales' products|.

Of all together, relative, for well spread inner rows: an error d of an inner
value whose codes are s apart changes its code with probability d / s, and then
by s, so the mean square of the change is d s; s is at most 2^-3 of the value,
which makes sqrt(0.1 d) of a relative error d.  32-bit sums: d = 2^-21 is
generous, 2.2e-4; twice that for a count of changes that is small.  The second
products add 5e-5 where they are 8-bit ones, f16 in between 2^-11 / sqrt(3):
``BESIDES``.  The result's rounding is at most 1 / sqrt(3) of its unit: ``NORM``.
"""

import numpy as np

from fp8_cut import cut8
from fp8_util import (BLOCK, ROUND, SMALLEST, TOP, block_values, blocks, code_values, quantize_interval, quantize_ref,
                      row_values)

ROOT3 = 3.0 ** 0.5
BESIDES = {"f32": 5e-4, "f16": 5e-4 + 5e-5, "bf16": 5e-4 + 5e-5 + 2.0 ** -11 / ROOT3}
NORM = {t: BESIDES[t] + ROUND[t] / ROOT3 for t in BESIDES}


def bound(x, ids, weights, layer, dtype):
    """(y, tolerance of each element) in 64 bits."""
    n, k = ids.shape
    hb, ib = blocks(layer.hidden), blocks(layer.inner)
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
        first = []
        for i in (0, 1):
            w = block_values(w13[e, i], s13[e, i], layer.hidden)
            first.append((xe @ w.T, np.abs(xe) @ np.abs(w).T * (BLOCK + hb + 8) * 2.0 ** -23))
        (g, dg), (u, du) = first
        with np.errstate(over="ignore"):
            silu = g / (1 + np.exp(-g))
        dh = 1.1 * dg * (np.abs(u) + du) + np.abs(silu) * du + np.abs(silu * u) * 2.0 ** -20
        hv, dv = quantize_interval(silu * u, dh)
        w = block_values(w2[e], s2[e], layer.inner)
        z, reach = hv @ w.T, (np.abs(hv) + dv) @ np.abs(w).T
        dz = dv @ np.abs(w).T + reach * (BLOCK + ib + 8) * 2.0 ** -23
        size = np.abs(silu * u) + dh
        most = np.maximum(np.stack([size[:, b:b + BLOCK].max(axis=1) for b in range(0, layer.inner, BLOCK)], axis=1),
                          2.0 ** -100) * 1.01
        if dtype != "f32":
            codes = np.zeros((len(token), ib * BLOCK))
            codes[:, :layer.inner] = hv / np.repeat(most / TOP, BLOCK, axis=1)[:, :layer.inner]
            dz = dz + 2 * cut8(codes, (most / TOP).T, w2[e], s2[e])
        if dtype == "bf16":
            total = (most / TOP) @ np.abs(s2[e].astype(np.float64)).T
            total = np.repeat(total, BLOCK, axis=1)[:, :layer.hidden]
            dz = dz + np.abs(z) * 2.0 ** -11 + total * TOP * TOP * BLOCK * 2.0 ** -39
        p = weights[token, slot].astype(np.float64)[:, None]
        np.add.at(y, token, z * p)
        np.add.at(tol, token, (dz + np.abs(z) * (k + 4) * 2.0 ** -23) * np.abs(p))
    return y, tol + np.abs(y) * ROUND[dtype] + SMALLEST[dtype]


def reference(x, ids, weights, layer):
    """y alone, for larger cases."""
    xq, xs = quantize_ref(x, 1)
    xv = row_values(xq, xs, layer.hidden)
    y = np.zeros((ids.shape[0], layer.hidden))
    w13, s13 = code_values(layer.w13), layer.w13_scale.cpu().numpy()
    w2, s2 = code_values(layer.w2), layer.w2_scale.cpu().numpy()
    for e in range(layer.experts):
        token, slot = np.nonzero(ids == e)
        if len(token) == 0:
            continue
        g, u = (xv[token] @ block_values(w13[e, i], s13[e, i], layer.hidden).T for i in (0, 1))
        with np.errstate(over="ignore"):
            h = (g / (1 + np.exp(-g)) * u).astype(np.float32)
        q, s = quantize_ref(h, 1)
        z = row_values(q, s, layer.inner) @ block_values(w2[e], s2[e], layer.inner).T
        np.add.at(y, token, z * weights[token, slot].astype(np.float64)[:, None])
    return y


def norm_error(y, ref):
    return float(np.linalg.norm(y.double().cpu().numpy() - ref) / np.linalg.norm(ref))
