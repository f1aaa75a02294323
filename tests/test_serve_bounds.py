"""The measure of a norm's mean error, on the kernels' steps and on coarser ones done by numpy; no GPU."""

import numpy as np
import pytest

from serve_bounds import RMS_ROUND

F, D = np.float32, np.float64


def rows_of_all_sizes(rows, cols, seed):
    """Rows whose root mean squares have mantissas all over [1, 2), logarithms uniform."""
    r = np.random.RandomState(seed)
    return (r.standard_normal((rows, cols)) * 2.0 ** r.uniform(-3, 3, (rows, 1))).astype(F)


def mean_error(y, ref):
    """Root mean square of the relative error."""
    return float(np.sqrt(np.mean(((y.astype(D) - ref) / ref) ** 2)))


def _thread_sums(x):
    """Chains of 16 fused steps: the product exact, each sum rounded once."""
    h = x.reshape(len(x), -1, 16)
    s = np.zeros(h.shape[:2], F)
    for i in range(16):
        s = (s.astype(D) + h[..., i].astype(D) ** 2).astype(F)
    return s


def _joined(s, kind):
    while s.shape[1] > 1:
        s = (s[:, 0::2].astype(kind) + s[:, 1::2].astype(kind)).astype(kind)
    return s


@pytest.mark.parametrize("join,root,fits", [(D, D, True), (F, F, False), (F, D, False), (D, F, False)])
def test_mean_error_tells_32_bits_from_64(join, root, fits):
    """Without gain a norm has two roundings that show, the factor's and the product's: 2^0.5 RMS_ROUND (the
    chains of 16, of which 128 are averaged, add a hundredth).  A join in 32 bits adds half of each step's, of which
    there are ever more and smaller ones: 1/4 (1 + 1/2 + 1/4 + ...) = 1/2 in the squares, 2.5^0.5 in all.  A mean, a sum
    with eps (half of each) and a root and quotient in 32 bits add 1/4 + 1/4 + 1 at least."""
    x = rows_of_all_sizes(2000, 2048, 1)
    ref = x.astype(D) / np.sqrt((x.astype(D) ** 2).mean(axis=1, keepdims=True) + D(F(1e-6)))
    total = _joined(_thread_sums(x), join)
    mean = (total.astype(root) / root(2048)).astype(root)
    factor = (root(1) / np.sqrt((mean + root(F(1e-6))).astype(root)).astype(root)).astype(F)
    err = mean_error(x * factor, ref)
    assert (err <= 1.05 * 2 ** 0.5 * RMS_ROUND) == fits, err / RMS_ROUND
