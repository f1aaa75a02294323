"""Norms, dense layers in 4 bits and sampling together: a layer's step as it is served, on streams, in graphs."""

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from fp8_util import (ROUND, SMALLEST, block_values, code_values, experts_ref, linear_tol, route_ref, row_values,
                      torch_dtype)
from gpu_util import device, note
from paper_1911_09723_amd.spconv import BF16
from serve_util import linear4_tol, norm_ref, norm_tol, quantize4_ref, sample_ref, to_numpy, unpacked, values4

pytestmark = pytest.mark.gpu


def _draw(rows, cols, dtype, seed, width=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, cols), generator=g) * width).to(torch_dtype(dtype)).to(device())


def _u(n, seed):
    import torch
    return torch.rand(n, generator=torch.Generator().manual_seed(seed)).to(device())


def _layer(dtype, batch, bits, seed=1, experts=8, hidden=320, inner=200, cout=1500, residual=True, **more):
    import torch
    g = torch.Generator().manual_seed(seed)

    def draw(*shape):
        return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device())

    nets = sp.Experts.from_dense(draw(experts, inner, hidden), draw(experts, inner, hidden),
                                 draw(experts, hidden, inner))
    head = (sp.Mxfp4Linear if bits == 4 else sp.Fp8Linear).from_dense(draw(cout, hidden) * 3, draw(cout))
    gains = [(1 + 0.2 * torch.randn(hidden, generator=g)).to(device()) for _ in range(2)]
    return sp.ExpertLayer(draw(experts, hidden) * 8, nets, 3, batch, torch_dtype(dtype), head, residual=residual,
                          norm=gains[0], head_norm=gains[1], eps=1e-5, **more)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("batch,bits,residual", [(1, 4, True), (13, 8, True), (40, 4, False), (70, 8, False), (200, 4, True)])
def test_steps_follow_each_other(dtype, batch, bits, residual):
    """Each step's output against the reference on what the step before left."""
    note("serving layer %s batch %d, %d bits" % (dtype, batch, bits))
    filters = dict(temperature=0.8, top_k=200, top_p=0.9)
    layer = _layer(dtype, batch, bits, residual=residual, sampler=filters)
    x, u = _draw(batch, 320, dtype, 2), _u(batch, 3)
    layer.u.copy_(u)
    out = layer.forward(x)
    r, xv = ROUND[dtype], to_numpy(x)
    # the norm that the router reads, and its rounding, which the experts read
    y, _ = norm_ref(xv, None, to_numpy(layer.norm), 1e-5)
    h32, h = to_numpy(layer.x32), to_numpy(layer.h)
    assert (np.abs(h32 - y) <= norm_tol(y, 320, "f32")).all()
    # (a value below the least normal one of the type, 2^-14 in float16, is off by up to half its spacing)
    assert (np.abs(h - h32) <= np.abs(h32) * r + SMALLEST[dtype] / 2).all()
    # router and experts
    logits, router = layer.logits.cpu().numpy(), to_numpy(layer.router)
    assert (np.abs(logits - h32 @ router.T) <= np.abs(h32) @ np.abs(router).T * 340 * 2.0 ** -24).all()
    ids, _ = route_ref(logits, 3)
    assert np.array_equal(layer.ids.cpu().numpy(), ids)
    e, tol = experts_ref(h.astype(np.float32), ids, layer.weights.cpu().numpy(), layer.experts, cut=dtype != "f32")
    total = to_numpy(layer.y)  # rounded once by the experts and once by the sum
    ref = e + xv if residual else e
    assert (np.abs(total - ref) <= tol + (np.abs(e) + np.abs(total)) * 1.01 * r + 1e-6).all()
    # The norm of the sum. The kernel norms the sum before its rounding, which moves an element by r of
    # itself, or half the spacing of the type's least values, and the root mean square by r of it at most.
    gain = to_numpy(layer.head_norm)
    y, _ = norm_ref(total, None, gain, 1e-5)
    moved = np.abs(y) * 2.02 * r + SMALLEST[dtype] * np.abs(gain) / np.sqrt((total * total).mean(axis=1, keepdims=True))
    if bits == 4:
        top = to_numpy(layer.top)
        assert (np.abs(top - y) <= norm_tol(y, 320, dtype) + moved).all()
        v = values4(*quantize4_ref(top), 320)
        w = values4(*unpacked(layer.head.w.cpu().numpy(), layer.head.w_scale.cpu().numpy()), 320)
        bound = linear4_tol
    else:
        v = row_values(code_values(layer.q), layer.q_scale.cpu().numpy(), 320)
        most = np.repeat(layer.q_scale.cpu().double().numpy().T * 448, 128, axis=1)[:, :320]
        # a code is half a step of e4m3 off (2^-4 of the value, or of the least normal one, 2^-6 of 448)
        assert (np.abs(v - y) <= np.abs(y) * (2.0 ** -4 + 2.0 ** -16) + most * 2.0 ** -6 / 448 * 2.0 ** -4 + 1.07 * moved).all()
        w = block_values(code_values(layer.head.w), layer.head.w_scale.cpu().numpy(), 320)
        bound = linear_tol
    b = to_numpy(layer.head.bias)
    ref = v @ w.T + b
    assert (np.abs(to_numpy(out) - ref) <= bound(ref, np.abs(v) @ np.abs(w).T + np.abs(b), 320, dtype)).all()
    # the tokens
    assert np.array_equal(layer.tokens.cpu().numpy(), sample_ref(to_numpy(out), u.cpu().numpy(), **filters))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("batch,cout", [(1, 1500), (50, 1500), (3, 20000)])
def test_replays_equal_eager_steps(batch, cout, bits):
    """Replays of a captured step with eager work between them, and the parameters of each row changed in place."""
    import torch
    note("replays of batch %d -> %d, %d bits" % (batch, cout, bits))
    t = torch.full((batch,), 0.9, device=device())
    ks = torch.full((batch,), 50, dtype=torch.int32, device=device())
    layer = _layer("bf16", batch, bits, cout=cout, sampler=dict(temperature=t, top_k=ks, top_p=0.95))
    layer.capture()
    for r in range(4):
        x, u = _draw(batch, 320, "bf16", 10 + r), _u(batch, 20 + r)
        t.fill_(0.5 + 0.3 * r)
        ks.fill_((50, 0, 3, 700)[r])
        layer.x.copy_(x)
        layer.u.copy_(u)
        out = layer.replay().clone()
        tokens = layer.tokens.clone()
        torch.cuda.synchronize()
        layer.tokens.fill_(-7)
        assert torch.equal(out, layer.forward(x)) and torch.equal(tokens, layer.tokens), "replay %d" % r
        layer.forward(_draw(batch, 320, "bf16", 90))
        torch.cuda.synchronize()


def test_layer_without_norms_is_as_before():
    """A 4-bit head and a sampler alone leave the layer's other steps as they were."""
    import torch
    a, b = (_layer("bf16", 9, bits) for bits in (4, 8))
    for layer in (a, b):
        layer.norm = layer.head_norm = None
    plain = sp.ExpertLayer(a.router, a.experts, 3, 9, torch.bfloat16)
    headed = sp.ExpertLayer(a.router, a.experts, 3, 9, torch.bfloat16, a.head, sampler=dict(temperature=0.0))
    x = _draw(9, 320, "bf16", 5)
    y = plain.forward(x).clone()
    out = headed.forward(x)
    assert torch.equal(headed.y, y) and torch.equal(out, a.head.run(y))
    assert np.array_equal(headed.tokens.cpu().numpy(), sample_ref(to_numpy(out), np.zeros(9), 0.0))


@pytest.mark.parametrize("bits", [4, 8])
def test_layers_whose_norms_are_taken_away(bits):
    """Without gains the layer's steps are those of its parts, called one by one; and of a layer made without any."""
    import torch
    note("layer without norms, %d bits" % bits)
    layer, x = _layer("bf16", 9, bits, sampler=dict(temperature=0.7, top_k=20)), _draw(9, 320, "bf16", 5)
    u = _u(9, 6)
    bare = sp.ExpertLayer(layer.router, layer.experts, 3, 9, torch.bfloat16, layer.head, sampler=layer.sampler)
    bare.u.copy_(u)
    out = bare.forward(x).clone()
    logits = torch.empty((9, 8), device=device())
    sp.spconv_linear(x.float(), layer.router, None, "none", logits, 9, 320, 8)
    total = layer.experts.run(x, *sp.route(logits, 3)) + x
    assert torch.equal(bare.y, total) and torch.equal(out, layer.head.run(total))
    assert torch.equal(bare.tokens, sp.sample(out, u, 0.7, 20))


def test_refusals_of_the_layer():
    import torch
    layer = _layer("bf16", 2, 4)
    args = (layer.router, layer.experts, 3, 2, torch.bfloat16)
    with pytest.raises(ValueError):
        sp.ExpertLayer(*args, head_norm=layer.head_norm)
    for bad in (layer.norm[:-1], layer.norm.cpu(), layer.norm.double()):
        with pytest.raises(ValueError):
            sp.ExpertLayer(*args, norm=bad)
        with pytest.raises(ValueError):
            sp.ExpertLayer(*args, layer.head, head_norm=bad)


def test_results_carry_no_gradient():
    """Inputs that require one are taken as they are; what comes out is cut off from them."""
    import torch
    x, gain = _draw(4, 256, "f32", 1).requires_grad_(), _draw(1, 256, "f32", 2)[0].requires_grad_()
    y, total = sp.rms_norm(x, gain, residual=x)
    head = sp.Mxfp4Linear.from_dense(_draw(300, 256, "f32", 3).requires_grad_())
    out = head.run(x)
    outs = (y, total, *sp.rms_norm_fp8(x, gain), *sp.quantize_mxfp4(x), out, sp.sample(x, _u(4, 4)))
    assert not any(o.requires_grad for o in outs)
    assert torch.equal(out, head.run(x.detach())) and torch.equal(y, sp.rms_norm(x.detach(), gain.detach(), residual=x.detach())[0])


def _calls(n, seed, spaces=None):
    """(a chain of every operator's calls with all that they write given, its outputs, its input, its workspaces)."""
    import torch
    dev, u8, f32 = device(), torch.uint8, torch.float32
    x, res, gain = _draw(n, 700, "bf16", seed), _draw(n, 700, "bf16", seed + 1), _draw(1, 700, "f32", seed + 2)[0]
    head = sp.Mxfp4Linear.from_dense(_draw(30000, 700, "f32", seed + 3))
    y, total = torch.empty_like(x), torch.empty_like(x)
    q8, s8 = torch.empty((n, 768), dtype=torch.float8_e4m3fn, device=dev), torch.empty((6, n), dtype=f32, device=dev)
    q4, s4 = torch.empty((n, 384), dtype=u8, device=dev), torch.empty((3, n, 8), dtype=u8, device=dev)
    out, out4 = (torch.empty((n, 30000), dtype=torch.bfloat16, device=dev) for _ in range(2))
    ids = torch.empty(n, dtype=torch.int32, device=dev)
    u, t = _u(n, seed + 4), torch.rand(n, device=dev) + 0.5
    if spaces is None:
        sizes = head.workspace_bytes(n, torch.bfloat16), sp.spconv_sample_workspace(BF16, n, 30000)
        spaces = [torch.empty(max(1, size), dtype=u8, device=dev) for size in sizes]
    linear_space, sample_space = spaces

    def step(stream=None):
        sp.rms_norm(x, gain, 1e-6, res, y=y, total=total, stream=stream)
        sp.rms_norm_fp8(x, gain, 1e-6, res, q=q8, scale=s8, total=total, stream=stream)
        sp.quantize_mxfp4(y, q4, s4, stream=stream)
        head.run(q4, s4, y=out4, stream=stream)
        head.run(y, y=out, workspace=linear_space, stream=stream)
        sp.sample(out, u, t, 300, 0.9, ids=ids, workspace=sample_space, stream=stream)

    return step, (y, total, q8.view(u8), s8, q4, s4, out4, out, ids), x, spaces


@pytest.mark.parametrize("n", [1, 20, 300])
def test_another_stream(n):
    """With outputs and workspaces given the calls run on a stream that is not torch's current one."""
    import torch
    note("another stream, %d rows" % n)
    step, outs, _, _ = _calls(n, 1)
    step()
    torch.cuda.synchronize()
    ref = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for o in outs:
        o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(o, r) for o, r in zip(outs, ref))


@pytest.mark.parametrize("n", [1, 50])
def test_two_streams_at_once(n):
    """Chains of calls on two streams, none waiting for the other, each with outputs and workspaces of its own."""
    import torch
    note("two streams, %d rows" % n)
    chains = [_calls(n, 1), _calls(n, 50)]
    refs = []
    for step, outs, _, _ in chains:
        step()
        torch.cuda.synchronize()
        refs.append([o.clone() for o in outs])
        for o in outs:
            o.zero_()
    sides = [torch.cuda.Stream() for _ in chains]
    for side in sides:
        side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for (step, _, _, _), side in zip(chains, sides):
            step(side)
    torch.cuda.synchronize()
    for (_, outs, _, _), ref in zip(chains, refs):
        assert all(torch.equal(o, r) for o, r in zip(outs, ref))


@pytest.mark.parametrize("n", [1, 33])
def test_two_graphs_share_workspaces(n):
    """Graphs of two calls' chains with the same workspaces, replayed in turn on one stream."""
    import torch
    note("two graphs, %d rows" % n)
    a = _calls(n, 1)
    chains = [a, _calls(n, 50, a[3])]
    graphs = []
    for step, _, _, _ in chains:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for r in range(4):
        for i, chain in enumerate(chains):
            chain[2].copy_(_draw(n, 700, "bf16", 100 + 10 * r + i))
        for space in a[3]:
            space.fill_(255 if r % 2 else 0)
        for o in chains[0][1] + chains[1][1]:
            o.zero_()
        for g in graphs:
            g.replay()
        got = [[o.clone() for o in outs] for _, outs, _, _ in chains]
        torch.cuda.synchronize()
        for (step, outs, _, _), g in zip(chains, got):
            step()
            assert all(torch.equal(o, v) for o, v in zip(outs, g)), "replay %d" % r
