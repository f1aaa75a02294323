"""Sampling where the number of kept tokens decides how they are found: around 512 and 1024, in long rows, with and without a share."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import torch_dtype
from gpu_util import device, note
from serve_util import sample_ref, to_numpy

pytestmark = pytest.mark.gpu

# a list in LDS holds 1024 tokens; alone, more than 512 are found by a histogram
COUNTS = [511, 512, 513, 700, 1000, 1023, 1024, 1025]
SHARES = [dict(), dict(top_p=0.9), dict(top_p=0.999, min_p=0.02), dict(top_p=0.3, temperature=0.6)]


def _rows(kind, n, vocab, dtype, seed):
    """Logits in which the border of k lies otherwise: spread out, among equal ones, with few tokens on, in one place."""
    import torch
    g = torch.Generator(device()).manual_seed(seed)
    x = torch.randn((n, vocab), generator=g, device=device()) * 2
    if kind == "ties":
        x = torch.round(x * 2) / 2
    elif kind == "flat":
        x = torch.where(x > 5, x, torch.zeros_like(x))
    elif kind == "masked":
        x[torch.rand((n, vocab), generator=g, device=device()) < 0.9] = -float("inf")
        x[0, 800:] = -float("inf")
        x[1, :-1] = float("nan")
    elif kind == "clustered":  # the largest side by side: a few segments hold all that is kept
        x[:, vocab // 3:vocab // 3 + 3000] += 40
    return x.to(torch_dtype(dtype))


def _compare(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    import torch
    ids = sp.sample(logits, u, temperature, top_k, top_p, min_p).cpu().numpy()
    host = [p.cpu().numpy() if torch.is_tensor(p) else p for p in (temperature, top_k, top_p, min_p)]
    ref = sample_ref(to_numpy(logits), u.cpu().numpy(), *host)
    assert np.array_equal(ids, ref), (np.flatnonzero(ids != ref), host)


@pytest.mark.parametrize("kind", ["spread", "ties", "flat", "masked", "clustered"])
@pytest.mark.parametrize("vocab,dtype", [(1000, "f32"), (8192, "bf16"), (8193, "f32"), (32000, "f16"), (50001, "f32"), (131072, "bf16"), (1 << 20, "bf16")])
def test_counts(vocab, dtype, kind):
    import torch
    n, long = (2, True) if vocab > 200000 else (4, False)
    for i, k in enumerate(COUNTS[1::3] + COUNTS[-2:] if long else COUNTS):
        for j, f in enumerate(SHARES[:2] if long else SHARES):
            note("sample %d x %d %s %s k = %d %s" % (n, vocab, dtype, kind, k, f))
            u = torch.rand(n, generator=torch.Generator().manual_seed(10 * i + j)).to(device())
            _compare(_rows(kind, n, vocab, dtype, 4 * i + j), u, top_k=k, **f)


@pytest.mark.parametrize("kind", ["spread", "ties", "clustered"])
@pytest.mark.parametrize("vocab,dtype", [(4000, "bf16"), (33000, "f32"), (131072, "bf16")])
def test_counts_by_row(vocab, dtype, kind):
    """All of them in one call, beside rows of other kinds."""
    import torch
    n = 40
    note("counts by row %d %s %s" % (vocab, dtype, kind))
    r = np.random.RandomState(vocab)
    t, p, m = (torch.tensor(r.choice(v, n), dtype=torch.float32, device=device()) for v in ([0.0, 0.5, 1.0, 1.3], [1.0, 1.0, 0.9, 0.99], [0.0, 0.0, 0.05]))
    k = torch.tensor(r.choice(COUNTS + [0, 1, 50, 2000], n), dtype=torch.int32, device=device())
    logits, u = _rows(kind, n, vocab, dtype, 7), torch.rand(n, generator=torch.Generator().manual_seed(8)).to(device())
    _compare(logits, u, t, k, p, m)
    _compare(logits, u, 0.9, k, 0.95, 0.0)
    _compare(logits, u, 0.9, k, 1.0, m)


@pytest.mark.parametrize("top_p", [1.0, 0.97])
def test_every_share_of_the_kept(top_p):
    """u from end to end over one row's kept tokens."""
    import torch
    logits = _rows("spread", 1, 20000, "f32", 9).expand(400, 20000).contiguous()
    u = (torch.arange(400, dtype=torch.float32) / 400).to(device())
    for k in COUNTS:
        note("shares k = %d p = %g" % (k, top_p))
        _compare(logits, u, 1.0, k, top_p)


def test_counts_in_a_graph():
    """A captured call whose counts change in place between replays."""
    import torch
    n, vocab = 9, 40000
    logits, u = _rows("spread", n, vocab, "bf16", 11), torch.rand(n, generator=torch.Generator().manual_seed(12)).to(device())
    k = torch.zeros(n, dtype=torch.int32, device=device())
    p = torch.ones(n, device=device())
    ids = torch.empty(n, dtype=torch.int32, device=device())
    space = torch.empty(sp.spconv_sample_workspace("bf16", n, vocab), dtype=torch.uint8, device=device())

    def step():
        sp.sample(logits, u, 0.9, k, p, ids=ids, workspace=space)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r, (count, share) in enumerate([(513, 1.0), (1024, 0.9), (1025, 0.9), (512, 1.0), (0, 0.9), (700, 0.5)]):
        note("replay %d" % r)
        k.fill_(count)
        p.fill_(share)
        ids.fill_(-7)
        graph.replay()
        got = ids.cpu().numpy()
        torch.cuda.synchronize()
        ref = sample_ref(to_numpy(logits), u.cpu().numpy(), 0.9, count, share)
        assert np.array_equal(got, ref), (count, share)
        logits.copy_(_rows("spread", n, vocab, "bf16", 20 + r))
