"""Workspaces stay within what a call needs at once; no GPU."""

import pytest

import paper_1911_09723_amd as sp

MOST = 1 << 20  # rows from here on are refused


@pytest.mark.parametrize("vocab", [8193, 8200, 32000, 131072, 1 << 20])
def test_sampling_of_many_rows_shares_its_workspace(vocab):
    """Rows that a launch does not take at once use the same space: it ends growing, long before it is as large as the logits."""
    size = sp.spconv_sample_workspace
    sizes = [size("bf16", n, vocab) for n in (1, 64, 1024, 4096, 32768, 100000, MOST - 1)]
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2] == sizes[-3]
    assert sizes[-1] <= 8192 * sizes[0] and sizes[-1] < 3 << 30
    assert sizes[2] == 1024 * sizes[0]


def test_short_rows_need_none():
    assert [sp.spconv_sample_workspace("f32", n, 8192) for n in (1, 5000, MOST - 1)] == [0, 0, 0]
