"""Bounds of norms and 4-bit products that count the kernels' own roundings, and 64-bit norms of long calls on the GPU."""

import numpy as np

from fp8_util import ROUND, SMALLEST
from serve_util import lines

UNIT = 2.0 ** -24  # half a step of float32, relative
# The relative error of one rounding to float32, root mean square: uniform within half a step,
# 2^-24 / m for a mantissa m in [1, 2) whose logarithm is uniform: 2^-24 sqrt(1/3) sqrt(E 1/m^2),
# E 1/m^2 = (1 - 1/4) / (2 ln 2) = 0.541.
RMS_ROUND = UNIT * (0.541 / 3) ** 0.5


def norm_chain(cols):
    """Most fused steps that one thread chains: 8 a piece, two pieces up to 16384 columns, four up to 32768, beyond one for each 8192."""
    return 16 if cols <= 16384 else 32 if cols <= 32768 else 8 * -(-cols // 8192)


def norm_bound(cols, residual):
    """Largest relative error of a norm in float32.  The sum: a step of the chain each, halved by the
    root; joining threads, mean and root are 64-bit.  Then the factor's rounding and two products.
    A residual's sum is rounded, once in the value and once (twice, halved) in the sum of squares."""
    return (norm_chain(cols) / 2 + 3 + (2 if residual else 0)) * UNIT * 1.01


def norm_tight(y, cols, dtype, residual):
    """The same with the rounding to y's type; y: a numpy array or a tensor in 64 bits."""
    return abs(y) * (norm_bound(cols, residual) + (0 if dtype == "f32" else ROUND[dtype] * 1.01)) + SMALLEST[dtype]


def norm64(x, residual=None, gain=None, eps=1e-6):
    """(y, h) of tensors, in 64 bits where they lie."""
    h = x.double() if residual is None else x.double() + residual.double()
    y = h / ((h * h).mean(dim=1, keepdim=True) + float(np.float32(eps))).sqrt()
    return (y if gain is None else y * gain.double()), h


def linear4_tight(y, terms, cin, dtype):
    """Two instructions a line of 256 channels, each at most 2^-22 of the magnitudes that it adds up (measured,
    2e-7), wherever a line's sum is carried; the sums of up to 16 wavefronts (no more than lines) and the bias
    by 32-bit additions; one rounding to the type."""
    n = lines(cin)
    return terms * (2 * n * 2.0 ** -22 + min(n, 16) * UNIT) * 1.01 + np.abs(y) * (0 if dtype == "f32" else ROUND[dtype] * 1.01) + SMALLEST[dtype]
