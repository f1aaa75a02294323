"""The next token from logits and given random numbers, against the definition in 64 bits."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import torch_dtype
from gpu_util import device, note
from serve_util import sample_ref, to_numpy

pytestmark = pytest.mark.gpu
INF = float("inf")


def _logits(n, vocab, dtype, seed, width=2.0, stride=None):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, vocab if stride is None else stride), generator=g) * width).to(torch_dtype(dtype)).to(device())[:, :vocab]


def _u(n, seed):
    import torch
    return torch.rand(n, generator=torch.Generator().manual_seed(seed)).to(device())


def _given(p, kind):
    import torch
    return torch.tensor(p, dtype=kind, device=device())


def _compare(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    import torch
    ids = sp.sample(logits, u, temperature, top_k, top_p, min_p)
    assert ids.dtype == torch.int32
    host = [p.cpu().numpy() if torch.is_tensor(p) else p for p in (temperature, top_k, top_p, min_p)]
    ref = sample_ref(to_numpy(logits), u.cpu().numpy(), *host)
    assert np.array_equal(ids.cpu().numpy(), ref), np.flatnonzero(ids.cpu().numpy() != ref)


FILTERS = [dict(), dict(temperature=0.0), dict(temperature=0.3), dict(temperature=3.0), dict(top_k=1), dict(top_k=40),
           dict(top_k=5000), dict(top_p=0.5), dict(top_p=0.95), dict(top_p=0.9999), dict(min_p=0.05), dict(top_k=50, top_p=0.9),
           dict(top_p=0.9, min_p=0.1), dict(top_k=30, min_p=0.2, temperature=0.7),
           dict(temperature=0.8, top_k=2000, top_p=0.97, min_p=0.01)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,vocab", [(5, 1), (4, 2), (7, 63), (3, 1000), (40, 4097), (2, 8191), (3, 8193), (9, 32000), (2, 50001), (3, 131072), (1, 1 << 20)])
def test_filters(n, vocab, dtype):
    for i, f in enumerate(FILTERS):
        note("sample %d x %d %s %s" % (n, vocab, dtype, f))
        _compare(_logits(n, vocab, dtype, i), _u(n, 50 + i), **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [0.0, 1e-3, 0.1, 10.0, 1000.0])
@pytest.mark.parametrize("vocab", [500, 20000, 70000])
def test_flat_and_steep_rows(vocab, width, dtype):
    for i, f in enumerate(FILTERS[::2]):
        note("width %g %d %s %s" % (width, vocab, dtype, f))
        _compare(_logits(6, vocab, dtype, 100 + i, width), _u(6, 150 + i), **f)


@pytest.mark.parametrize("vocab", [700, 33000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_parameters_by_row(vocab, dtype):
    import torch
    n = 64
    note("by row %d %s" % (vocab, dtype))
    r = np.random.RandomState(1)
    t = _given(r.choice([0.0, 0.2, 0.7, 1.0, 2.0], n), torch.float32)
    k = _given(r.choice([0, 1, 3, 50, 400, vocab, vocab + 9], n), torch.int32)
    p = _given(r.choice([0.0, 0.3, 0.9, 0.99, 1.0], n), torch.float32)
    m = _given(r.choice([0.0, 0.01, 0.3, 1.0], n), torch.float32)
    logits, u = _logits(n, vocab, dtype, 2), _u(n, 3)
    _compare(logits, u, t, k, p, m)
    _compare(logits, u, t, 50, p, 0.0)
    _compare(logits, u, 0.9, k, 1.0, m)


def test_parameters_out_of_their_ranges():
    """On the device they count as the header says."""
    import torch
    nan = float("nan")
    logits = _logits(12, 3000, "f32", 4)
    u = _given([-1.0, nan, 1.0, 5.0, 0.0, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.9999999], torch.float32)
    t = _given([1, 1, 1, 1, 1, -2.0, nan, 1, 1, 1, 1, INF], torch.float32)
    k = _given([0, 0, 0, 0, 0, 0, 0, -5, 1 << 30, 0, 0, 0], torch.int32)
    p = _given([1, 1, 1, 1, 1, 1, 1, 1, nan, -1.0, 7.0, 1], torch.float32)
    m = _given([0, 0, 0, 0, 0, 0, 0, 0, 0, nan, -1.0, 0], torch.float32)
    _compare(logits, u, t, k, p, m)
    _compare(logits, u, 1.0, 0, 1.0, _given([9.0] * 12, torch.float32))
    assert sp.sample(logits, u, t, k, p, m)[9].item() == logits[9].argmax().item()


@pytest.mark.parametrize("vocab", [1000, 40000])
def test_temperatures_of_every_size(vocab):
    """From the smallest float, where the largest logit takes all, to infinity, where tokens weigh the same."""
    import torch
    each = [1e-45, 1e-38, 1e-10, 1e-3, 30.0, 1e10, 3e38, INF]
    logits, u = _logits(8, vocab, "f32", 21), _u(8, 22)
    logits[:, 7] = 3e38 if vocab > 20000 else 5.0
    for f in (dict(), dict(top_k=30), dict(top_p=0.9), dict(min_p=0.5), dict(top_k=600)):
        note("temperatures %d %s" % (vocab, f))
        _compare(logits, u, _given(each, torch.float32), f.get("top_k", 0), f.get("top_p", 1.0), f.get("min_p", 0.0))
        for t in each:
            _compare(logits[:2], u[:2], t, **f)


@pytest.mark.parametrize("vocab", [1000, 40000])
def test_distances_past_the_largest_float(vocab):
    """Logits of both ends of float32: their distance is infinite there, and they weigh the same where t is."""
    logits = _logits(6, vocab, "f32", 31)
    logits[:, 5:vocab // 2] = -3e38
    logits[:, vocab - 7] = 3e38
    logits[2:4, 9:90] = -INF
    u = _u(6, 32)
    for t in (INF, 3e38, 1e37, 1.0):
        for f in (dict(), dict(top_k=vocab // 4), dict(top_k=vocab - 3), dict(top_p=0.3), dict(top_p=0.999999), dict(min_p=0.5),
                  dict(top_k=vocab - 100, top_p=0.9)):
            note("distances %d t = %g %s" % (vocab, t, f))
            _compare(logits, u, t, **f)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [1000, 40000])
def test_masked_tokens(vocab, dtype):
    """Off tokens, rows with one token or none, the type's lowest value, infinities and NaN."""
    import torch
    note("masked %d %s" % (vocab, dtype))
    kind = torch_dtype(dtype)
    low = torch.finfo(kind).min
    base = _logits(10, vocab, dtype, 5).clone()
    base[0] = -INF
    base[1] = float("nan")
    base[2] = -INF
    base[2, vocab - 1] = -3.0
    base[3, ::2] = -INF
    base[4, ::3] = float("nan")
    base[5] = low
    base[6, 1:] = low
    base[7, 17], base[7, vocab - 2] = INF, INF
    base[8] = torch.where(torch.arange(vocab, device=device()) % 5 == 0, base[8], torch.tensor(low, dtype=kind, device=device()))
    base[9, :vocab // 2] = -INF
    for i, f in enumerate(FILTERS):
        _compare(base, _u(10, 60 + i), **f)
    assert sp.sample(base, _u(10, 1)).cpu().tolist()[:3] == [-1, -1, vocab - 1]


@pytest.mark.parametrize("vocab", [100, 9000, 30000])
def test_equal_logits_go_by_index(vocab):
    """Signed zeros are equal; of a tie at a filter's border the lower indices stay."""
    import torch
    x = torch.zeros((8, vocab), device=device())
    x[:, ::2] = -0.0
    u = _given([0.0, 0.1, 0.25, 0.5, 0.5, 0.75, 0.9, 0.99], torch.float32)
    _compare(x, u)
    _compare(x, u, top_k=8)
    assert sp.sample(x, u, top_k=8).cpu().tolist() == [0, 0, 2, 4, 4, 6, 7, 7]
    _compare(x, u, top_p=0.5)
    assert sp.sample(x, u, 0.0).cpu().tolist() == [0] * 8
    x[:, vocab // 3:] += 1.0
    x[:, vocab - 7] = 2.0
    for f in FILTERS:
        _compare(x, u, **f)


def test_numbers_at_the_ends():
    """u = 0 takes the first kept token, however small its weight; the largest u the last of weight."""
    import torch
    x = torch.zeros((2, 5000), device=device())
    x[:, 2500] = 60.0  # the others weigh 1e-26
    u = _given([0.0, 1 - 2.0 ** -24], torch.float32)
    assert sp.sample(x, u).cpu().tolist() == [0, 2500]
    assert sp.sample(x, u, top_k=1).cpu().tolist() == [2500, 2500]
    x[:, 2500] = 0.0
    assert sp.sample(x, u).cpu().tolist() == [0, 4999]


def test_every_u_of_a_small_row():
    """The shares of all tokens, by a walk over u that meets each border's both sides."""
    import torch
    logits = _logits(1, 37, "f32", 9).repeat(4096, 1)
    u = (torch.arange(4096, dtype=torch.float32) / 4096).to(device())
    _compare(logits, u)
    _compare(logits, u, 0.6, 20, 0.93, 0.01)


def test_strided_rows_and_given_outputs():
    import torch
    for vocab, stride in ((1000, 1003), (33001, 33010)):
        logits, u = _logits(6, vocab, "bf16", 10, stride=stride), _u(6, 11)
        for f in FILTERS[::3]:
            _compare(logits, u, **f)
        ids = torch.full((8,), 99, dtype=torch.int32, device=device())
        size = sp.spconv_sample_workspace("bf16", 6, vocab)
        space = torch.full((size + 64,), 7, dtype=torch.uint8, device=device())
        out = sp.sample(logits, u, 0.7, 20, 0.9, ids=ids[1:7], workspace=space)
        assert out.data_ptr() == ids[1:7].data_ptr() and ids[0] == 99 and ids[7] == 99
        assert torch.equal(out, sp.sample(logits, u, 0.7, 20, 0.9)) and (space[size:] == 7).all()


def test_the_workspace_may_hold_anything():
    """Whatever an earlier call or another program left there."""
    import torch
    n, vocab = 5, 60000
    logits, u = _logits(n, vocab, "f32", 12), _u(n, 13)
    size = sp.spconv_sample_workspace("f32", n, vocab)
    for f in FILTERS[::2]:
        first = sp.sample(logits, u, **f)
        for fill in (0, 255, 127):
            space = torch.full((size + 16,), fill, dtype=torch.uint8, device=device())
            for _ in range(2):
                assert torch.equal(sp.sample(logits, u, **f, workspace=space), first), (f, fill)


def test_same_choice_in_every_call():
    import torch
    logits, u = _logits(30, 70000, "f32", 14), _u(30, 15)
    first = sp.sample(logits, u, 0.9, 0, 0.99)
    assert all(torch.equal(sp.sample(logits, u, 0.9, 0, 0.99), first) for _ in range(20))
    parts = torch.cat([sp.sample(logits[i:i + 1], u[i:i + 1], 0.9, 0, 0.99) for i in range(30)])
    assert torch.equal(parts, first)


def test_rows_past_32_bit_offsets():
    import torch
    logits = torch.empty((2, 3 << 30), dtype=torch.float16, device=device())[:, :40000]
    logits.copy_(_logits(2, 40000, "f16", 16))
    u = _u(2, 17)
    for f in FILTERS[::4]:
        assert torch.equal(sp.sample(logits, u, **f), sp.sample(logits.contiguous(), u, **f))


def test_more_rows_than_a_launch():
    """Rows past 32768 of more than one chunk, with parameters by row."""
    import torch
    n, vocab = 32773, 8200
    logits = torch.randn((n, vocab), device=device(), generator=torch.Generator(device()).manual_seed(41)).half()
    u = torch.rand(n, device=device(), generator=torch.Generator(device()).manual_seed(42))
    t = torch.linspace(0.0, 2.0, n, device=device())
    k = (torch.arange(n, device=device()) % 7 * 30).int()
    p = torch.where(torch.arange(n, device=device()) % 3 == 0, 0.9, 1.0)
    ids = sp.sample(logits, u, t, k, p)
    for rows in (slice(0, 40), slice(32750, 32773)):
        some = sample_ref(*(to_numpy(v[rows]) for v in (logits, u, t)), k[rows].cpu().numpy(), to_numpy(p[rows]))
        assert np.array_equal(ids[rows].cpu().numpy(), some)
    for f in (dict(), dict(temperature=0.0), dict(top_k=20)):
        ids = sp.sample(logits, u, **f)
        assert torch.equal(ids[32700:], sp.sample(logits[32700:], u[32700:], **f))


def test_no_rows_and_refusals():
    import torch
    assert sp.sample(torch.empty((0, 9), device=device()), torch.empty(0, device=device())).shape == (0,)
    x, u = torch.zeros((3, 50), device=device()), torch.zeros(3, device=device())
    for call in (lambda: sp.sample(x, 0.5), lambda: sp.sample(x, u[:2]), lambda: sp.sample(x, u.cpu()),
                 lambda: sp.sample(x, u.double()), lambda: sp.sample(x[0], u), lambda: sp.sample(x[:, ::2], u),
                 lambda: sp.sample(x, u, u[:2]), lambda: sp.sample(x, u, top_k=u), lambda: sp.sample(x, u, top_p=u.half()),
                 lambda: sp.sample(x, u, ids=u), lambda: sp.sample(x, u, top_k=(1 << 32) + 5), lambda: sp.sample(x, u, min_p=torch.zeros((3, 1), device=device()))):
        with pytest.raises(ValueError):
            call()
    for f in (dict(temperature=-1.0), dict(top_k=-1), dict(top_p=1.1), dict(min_p=-0.5), dict(temperature=float("nan"))):
        with pytest.raises(sp.SpconvError):
            sp.sample(x, u, **f)
