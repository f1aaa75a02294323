"""What the 8-bit products, the router and the experts refuse, and their
workspace sizes; no GPU: every check on the arguments runs before any HIP call,
and no call here passes them all with work to do."""

import ctypes

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from paper_1911_09723_amd import spconv as S

A, B, C, D, E_, F = (1 << 40, 2 << 40, 3 << 40, 4 << 40, 5 << 40, 6 << 40)  # addresses that nothing reads
G, H, I = 7 << 40, 8 << 40, 9 << 40


def _quantize(**kw):
    a = dict(x=A, dtype="f32", ldx=300, rows=5, cols=300, block_rows=1, q=B, scale=C)
    a.update(kw)
    return sp.spconv_quantize_fp8(a["x"], a["dtype"], a["ldx"], a["rows"], a["cols"], a["block_rows"], a["q"],
                                  a["scale"], stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), S.E_ARG), (dict(q=None), S.E_ARG), (dict(scale=None), S.E_ARG), (dict(rows=-1), S.E_ARG),
    (dict(cols=-1), S.E_ARG), (dict(ldx=299), S.E_ARG), (dict(dtype=3), S.E_ARG), (dict(dtype=9), S.E_ARG),
    (dict(block_rows=64), S.E_UNSUPPORTED), (dict(block_rows=0), S.E_UNSUPPORTED),
    (dict(rows=1 << 26, cols=257, ldx=257), S.E_SHAPE), (dict(rows=1, cols=(1 << 30) + 1, ldx=1 << 31), S.E_SHAPE),
    (dict(ldx=1 << 40), S.E_SHAPE), (dict(x=A + 2), S.E_ARG), (dict(q=B + 8), S.E_ARG), (dict(scale=C + 1), S.E_ARG),
    (dict(q=A + 16), S.E_ARG), (dict(scale=B + 64), S.E_ARG), (dict(scale=A + 5 * 300 * 4 - 4), S.E_ARG),
])
def test_quantize_refuses(kw, status):
    assert _quantize(**kw) == status and sp.spconv_last_error()


@pytest.mark.parametrize("kw", [dict(rows=0), dict(cols=0, ldx=0), dict(rows=0, x=None, q=None, scale=None)])
def test_quantize_of_nothing(kw):
    assert _quantize(**kw) == S.OK


def _linear(**kw):
    a = dict(x=A, x_dtype="bf16", ldx=300, x_scale=None, w=B, w_scale=C, bias=D, act="relu", y=E_, y_dtype="bf16",
             n=100, cin=300, cout=200, ws=F, size=1 << 30)
    a.update(kw)
    return sp.spconv_linear_fp8(a["x"], a["x_dtype"], a["ldx"], a["x_scale"], a["w"], a["w_scale"], a["bias"],
                                a["act"], a["y"], a["y_dtype"], a["n"], a["cin"], a["cout"], a["ws"], a["size"],
                                stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), S.E_ARG), (dict(w=None), S.E_ARG), (dict(w_scale=None), S.E_ARG), (dict(y=None), S.E_ARG),
    (dict(n=-1), S.E_ARG), (dict(cin=-1), S.E_ARG), (dict(cout=-1), S.E_ARG), (dict(x_dtype=4), S.E_ARG),
    (dict(y_dtype="fp8"), S.E_ARG), (dict(act=3), S.E_ARG), (dict(ldx=299), S.E_ARG), (dict(x_scale=G), S.E_ARG),
    (dict(x_dtype="fp8"), S.E_ARG), (dict(cin=0), S.E_SHAPE), (dict(cin=(1 << 22) + 1, ldx=1 << 23), S.E_SHAPE),
    (dict(n=1 << 26, cin=300, cout=1), S.E_SHAPE), (dict(n=1 << 20, cin=1, cout=1 << 17), S.E_SHAPE),
    (dict(ws=None), S.E_ARG), (dict(size=100), S.E_ARG), (dict(ws=F + 8), S.E_ARG), (dict(w=B + 8), S.E_ARG),
    (dict(x=A + 1), S.E_ARG), (dict(y=E_ + 1), S.E_ARG), (dict(bias=D + 2), S.E_ARG), (dict(y=A), S.E_ARG),
    (dict(y=B + 32), S.E_ARG), (dict(ws=E_), S.E_ARG), (dict(ws=C), S.E_ARG), (dict(y=D), S.E_ARG),
    (dict(x_dtype="fp8", x_scale=G, x=A + 8), S.E_ARG), (dict(x_dtype="fp8", x_scale=E_), S.E_ARG),
    (dict(ldx=1 << 40), S.E_SHAPE),
])
def test_linear_refuses(kw, status):
    assert _linear(**kw) == status and sp.spconv_last_error()


@pytest.mark.parametrize("kw", [dict(n=0), dict(cout=0), dict(n=0, x=None, w=None, y=None, ws=None)])
def test_linear_of_nothing(kw):
    assert _linear(**kw) == S.OK


def test_linear_workspace():
    size = sp.spconv_linear_fp8_workspace
    assert size("fp8", 1000, 4096, 4096) == 0
    assert size("bf16", 1, 4096, 4096) == 0
    assert size("bf16", 1000, 300, 64) == 1000 * 384 + 1000 * 3 * 4
    assert size("f32", 0, 300, 64) == 0
    with pytest.raises(sp.SpconvError):
        size("bf16", 10, 0, 64)
    assert S.load_library().spconv_linear_fp8_workspace(0, 1, 1, 1, None) == S.E_ARG


def _route(**kw):
    a = dict(logits=A, dtype="f32", ld=64, bias=B, score="softmax", n=10, experts=64, groups=8, groups_kept=4,
             group_top=2, k=6, renorm=True, factor=1.0, ids=C, weights=D)
    a.update(kw)
    return sp.spconv_route(a["logits"], a["dtype"], a["ld"], a["bias"], a["score"], a["n"], a["experts"], a["groups"],
                           a["groups_kept"], a["group_top"], a["k"], a["renorm"], a["factor"], a["ids"],
                           a["weights"], stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), S.E_ARG), (dict(ids=None), S.E_ARG), (dict(weights=None), S.E_ARG), (dict(n=-1), S.E_ARG),
    (dict(k=0), S.E_ARG), (dict(groups=0), S.E_ARG), (dict(groups_kept=0), S.E_ARG), (dict(groups_kept=9), S.E_ARG),
    (dict(score=2), S.E_ARG), (dict(dtype="fp8"), S.E_ARG), (dict(ld=63), S.E_ARG), (dict(groups=7), S.E_SHAPE),
    (dict(k=65, experts=64), S.E_SHAPE), (dict(experts=2048, ld=2048), S.E_UNSUPPORTED),
    (dict(experts=130, groups=65, ld=130), S.E_UNSUPPORTED), (dict(experts=128, ld=128, k=65), S.E_UNSUPPORTED),
    (dict(group_top=3), S.E_UNSUPPORTED), (dict(group_top=0), S.E_UNSUPPORTED), (dict(n=1 << 25), S.E_SHAPE),
    (dict(logits=A + 2), S.E_ARG), (dict(ids=C + 2), S.E_ARG), (dict(ids=A + 64), S.E_ARG),
    (dict(weights=C + 4), S.E_ARG), (dict(weights=B), S.E_ARG), (dict(ld=1 << 40), S.E_SHAPE),
])
def test_route_refuses(kw, status):
    assert _route(**kw) == status and sp.spconv_last_error()


def test_route_of_nothing():
    assert _route(n=0, logits=None, ids=None, weights=None) == S.OK


def _experts(**kw):
    a = dict(x=A, dtype="bf16", ldx=256, ids=B, weights=C, w13=D, s13=E_, w2=F, s2=G, y=H, n=20, k=2, experts=8,
             hidden=256, inner=128, ws=I, size=1 << 30)
    a.update(kw)
    return sp.spconv_experts_fp8(a["x"], a["dtype"], a["ldx"], a["ids"], a["weights"], a["w13"], a["s13"], a["w2"],
                                 a["s2"], a["y"], a["n"], a["k"], a["experts"], a["hidden"], a["inner"], a["ws"],
                                 a["size"], stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), S.E_ARG), (dict(ids=None), S.E_ARG), (dict(weights=None), S.E_ARG), (dict(w13=None), S.E_ARG),
    (dict(s13=None), S.E_ARG), (dict(w2=None), S.E_ARG), (dict(s2=None), S.E_ARG), (dict(y=None), S.E_ARG),
    (dict(ws=None), S.E_ARG), (dict(n=-1), S.E_ARG), (dict(k=0), S.E_ARG), (dict(experts=0), S.E_SHAPE),
    (dict(hidden=0), S.E_SHAPE), (dict(inner=0), S.E_SHAPE), (dict(ldx=255), S.E_ARG), (dict(dtype="fp8"), S.E_ARG),
    (dict(experts=1025), S.E_UNSUPPORTED), (dict(k=65), S.E_UNSUPPORTED), (dict(hidden=32769, ldx=32769), S.E_UNSUPPORTED),
    (dict(inner=32769), S.E_UNSUPPORTED), (dict(n=1 << 23, k=4), S.E_SHAPE), (dict(n=1 << 17, inner=32768), S.E_SHAPE),
    (dict(size=1000), S.E_ARG), (dict(ws=I + 8), S.E_ARG), (dict(w13=D + 8), S.E_ARG), (dict(x=A + 1), S.E_ARG),
    (dict(ids=B + 2), S.E_ARG), (dict(y=A), S.E_ARG), (dict(y=F + 256), S.E_ARG), (dict(ws=H), S.E_ARG),
    (dict(ws=B), S.E_ARG), (dict(y=C), S.E_ARG), (dict(ldx=1 << 40), S.E_SHAPE),
])
def test_experts_refuse(kw, status):
    assert _experts(**kw) == status and sp.spconv_last_error()


def test_experts_of_nothing():
    assert _experts(n=0, x=None, y=None, ws=None) == S.OK


def test_experts_workspace():
    """Grows with the tokens, holds every piece that a call lays out, and is refused as the call is."""
    size = sp.spconv_experts_fp8_workspace
    assert size(0, 2, 8, 256, 128) == 0
    one = size(1, 2, 8, 256, 128)
    assert one >= 2 * 128 * 4
    n, k, e, h, i = 100, 2, 8, 300, 200
    pairs = n * k
    pieces = (2 * pairs * 4 + (e + 1) * 4 + n * 384 + n * 3 * 4 + pairs * 256 + pairs * 2 * 4 + pairs * h * 4 +
              pairs * 3 * 4)
    assert pieces <= size(n, k, e, h, i) <= pieces + 16 * 256
    sizes = [size(n, 2, 8, 256, 128) for n in range(3, 400, 7)]
    assert sizes == sorted(sizes)
    with pytest.raises(sp.SpconvError):
        size(1, 0, 8, 256, 128)
    assert S.load_library().spconv_experts_fp8_workspace(1, 1, 1, 1, 1, None) == S.E_ARG


def test_bf16_and_fp8_are_no_plan_storage():
    """The new element types belong to the new operators only."""
    for storage in (S.BF16, S.FP8):
        status, plan = sp.spconv_plan_create(4, 4, 1, np.zeros(5, np.int32), np.zeros(1, np.int32),
                                             np.zeros(1, np.float32), storage=storage, check=False)
        assert status == S.E_ARG and not plan


def test_python_wrappers_refuse_host_tensors_and_wrong_shapes():
    import torch
    x = torch.zeros(4, 128)
    for call in (lambda: sp.quantize_fp8(x), lambda: sp.route(x, 2),
                 lambda: sp.Fp8Linear(torch.zeros(4, 128).to(torch.float8_e4m3fn), torch.ones(1, 1), 4, 128),
                 lambda: sp.Experts(torch.zeros(1, 2, 4, 128).to(torch.float8_e4m3fn), torch.ones(1, 2, 1, 1),
                                    torch.zeros(1, 128, 128).to(torch.float8_e4m3fn), torch.ones(1, 1, 1), 128, 4),
                 lambda: sp.quantize_fp8(x.long()), lambda: sp.quantize_fp8(x[0])):
        with pytest.raises(ValueError):
            call()


def test_messages_and_status_of_the_last_call():
    assert _route(k=0) == S.E_ARG and "k" in sp.spconv_last_error()
    assert _route(n=0) == S.OK and sp.spconv_last_error() == ""


def test_library_takes_the_declared_arguments():
    """Every argument of the binding is one of the header's (name and count)."""
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "spconv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    lib = S.load_library()
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float,
             "spconv_dtype": ctypes.c_int32, "spconv_act": ctypes.c_int32, "spconv_score": ctypes.c_int32}
    for name in ("spconv_quantize_fp8", "spconv_linear_fp8", "spconv_linear_fp8_workspace", "spconv_route",
                 "spconv_experts_fp8", "spconv_experts_fp8_workspace"):
        args = re.search(name + r"\(([^)]*)\)", text).group(1).split(",")
        declared = getattr(lib, name).argtypes
        assert len(args) == len(declared), name
        for arg, kind in zip(args, declared):
            pointer = "*" in arg
            if not pointer:
                assert kind is kinds[arg.split()[0]], (name, arg)
            else:
                assert kind is ctypes.c_void_p or issubclass(kind, ctypes._Pointer), (name, arg)
