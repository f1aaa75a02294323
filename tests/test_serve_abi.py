"""What norms, 4-bit products and sampling refuse, and their workspace sizes; no
GPU: every check on the arguments runs before any HIP call, and no call here
passes them all with work to do."""

import ctypes
import os
import re

import numpy as np
import pytest

import paper_1911_09723_amd as sp
from paper_1911_09723_amd import spconv as S
from serve_util import e2m1, quantize4_ref, sample_ref, unpacked, packed, values4

A, B, C, D, E_, F, G, H, I, J = (i << 40 for i in range(1, 11))  # addresses that nothing reads
NAN, INF = float("nan"), float("inf")


def _norm(**kw):
    a = dict(x=A, dtype="bf16", ldx=300, residual=B, residual_dtype="bf16", ldr=300, total=C, ldt=300, gain=D,
             gain_dtype="bf16", eps=1e-6, y=E_, y_dtype="bf16", ldy=300, q=F, scale=G, rows=5, cols=300)
    a.update(kw)
    return sp.spconv_rms_norm(*a.values(), stream=0, check=False)


BAD_NORMS = [
    (dict(x=None), S.E_ARG), (dict(y=None, q=None, scale=None), S.E_ARG), (dict(q=None), S.E_ARG),
    (dict(scale=None), S.E_ARG), (dict(residual=None), S.E_ARG), (dict(rows=-1), S.E_ARG), (dict(cols=-1), S.E_ARG),
    (dict(dtype="fp8"), S.E_ARG), (dict(dtype=9), S.E_ARG), (dict(residual_dtype=3), S.E_ARG),
    (dict(gain_dtype=4), S.E_ARG), (dict(y_dtype=-1), S.E_ARG), (dict(residual_dtype="f16"), S.E_UNSUPPORTED),
    (dict(gain_dtype="f16"), S.E_UNSUPPORTED), (dict(y_dtype="f16"), S.E_UNSUPPORTED),
    (dict(dtype="f32", ldx=300, gain_dtype="f32", y_dtype="f32"), S.E_UNSUPPORTED),
    (dict(eps=-1e-6), S.E_ARG), (dict(eps=NAN), S.E_ARG), (dict(eps=INF), S.E_ARG), (dict(ldx=299), S.E_ARG),
    (dict(ldr=299), S.E_ARG), (dict(ldt=299), S.E_ARG), (dict(ldy=299), S.E_ARG),
    (dict(rows=1 << 26), S.E_SHAPE), (dict(rows=1 << 25, cols=64), S.E_SHAPE), (dict(ldx=1 << 40), S.E_SHAPE), (dict(ldr=1 << 40), S.E_SHAPE),
    (dict(ldt=1 << 40), S.E_SHAPE), (dict(ldy=1 << 40), S.E_SHAPE), (dict(x=A + 1), S.E_ARG),
    (dict(residual=B + 1), S.E_ARG), (dict(total=C + 1), S.E_ARG), (dict(gain=D + 1), S.E_ARG),
    (dict(y=E_ + 1), S.E_ARG), (dict(q=F + 8), S.E_ARG), (dict(scale=G + 2), S.E_ARG),
    # in the place of an input, but not exactly: another address, stride or element size
    (dict(total=B + 2), S.E_ARG), (dict(total=A + 2), S.E_ARG), (dict(total=B, ldt=301), S.E_ARG),
    (dict(y=A + 600), S.E_ARG), (dict(y=B, y_dtype="f32"), S.E_ARG), (dict(y=A, ldy=304), S.E_ARG),
    (dict(total=E_), S.E_ARG), (dict(total=B, y=B), S.E_ARG), (dict(total=D), S.E_ARG), (dict(y=D), S.E_ARG),
    (dict(q=A), S.E_ARG), (dict(q=E_), S.E_ARG), (dict(scale=C), S.E_ARG), (dict(q=G), S.E_ARG), (dict(q=D), S.E_ARG),
]


@pytest.mark.parametrize("kw,status", BAD_NORMS)
def test_norm_refuses(kw, status):
    assert _norm(**kw) == status and sp.spconv_last_error()


@pytest.mark.parametrize("kw", [dict(rows=0), dict(cols=0, ldx=0, ldr=0, ldt=0, ldy=0),
                                dict(rows=0, x=None, residual=None, total=None, y=None, q=None, scale=None)])
def test_norm_of_nothing(kw):
    assert _norm(**kw) == S.OK


def _quantize(**kw):
    a = dict(x=A, dtype="f32", ldx=300, rows=5, cols=300, q=B, scale=C)
    a.update(kw)
    return sp.spconv_quantize_mxfp4(*a.values(), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), S.E_ARG), (dict(q=None), S.E_ARG), (dict(scale=None), S.E_ARG), (dict(rows=-1), S.E_ARG),
    (dict(cols=-1), S.E_ARG), (dict(ldx=299), S.E_ARG), (dict(dtype="fp8"), S.E_ARG), (dict(dtype="mxfp4"), S.E_ARG),
    (dict(rows=1 << 24, cols=4097, ldx=5000), S.E_SHAPE), (dict(rows=1 << 25), S.E_SHAPE), (dict(rows=1, cols=(1 << 30) + 1, ldx=1 << 31), S.E_SHAPE),
    (dict(ldx=1 << 40), S.E_SHAPE), (dict(x=A + 2), S.E_ARG), (dict(q=B + 8), S.E_ARG), (dict(scale=C + 8), S.E_ARG),
    (dict(q=A + 16), S.E_ARG), (dict(scale=B + 64), S.E_ARG), (dict(scale=A + 5 * 300 * 4 - 16), S.E_ARG),
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
    return sp.spconv_linear_mxfp4(*a.values(), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), S.E_ARG), (dict(w=None), S.E_ARG), (dict(w_scale=None), S.E_ARG), (dict(y=None), S.E_ARG),
    (dict(n=-1), S.E_ARG), (dict(cin=-1), S.E_ARG), (dict(cout=-1), S.E_ARG), (dict(x_dtype="fp8"), S.E_ARG),
    (dict(y_dtype="mxfp4"), S.E_ARG), (dict(act=3), S.E_ARG), (dict(ldx=299), S.E_ARG), (dict(x_scale=G), S.E_ARG),
    (dict(x_dtype="mxfp4"), S.E_ARG), (dict(cin=0), S.E_SHAPE), (dict(cin=(1 << 22) + 1, ldx=1 << 23), S.E_SHAPE),
    (dict(n=1 << 25, cin=1, cout=1), S.E_SHAPE), (dict(n=1 << 24, cin=2049, ldx=2049, cout=1), S.E_SHAPE), (dict(n=1 << 20, cin=1, cout=1 << 17), S.E_SHAPE),
    (dict(n=1, cin=1 << 22, ldx=1 << 22, cout=1 << 14), S.E_SHAPE), (dict(ldx=1 << 40), S.E_SHAPE),
    (dict(ws=None), S.E_ARG), (dict(size=100), S.E_ARG), (dict(ws=F + 8), S.E_ARG), (dict(w=B + 8), S.E_ARG),
    (dict(w_scale=C + 8), S.E_ARG), (dict(x=A + 1), S.E_ARG), (dict(y=E_ + 1), S.E_ARG), (dict(bias=D + 2), S.E_ARG),
    (dict(y=A), S.E_ARG), (dict(y=B + 32), S.E_ARG), (dict(ws=E_), S.E_ARG), (dict(ws=C), S.E_ARG), (dict(y=D), S.E_ARG),
    (dict(x_dtype="mxfp4", x_scale=G, x=A + 8), S.E_ARG), (dict(x_dtype="mxfp4", x_scale=G + 8), S.E_ARG),
    (dict(x_dtype="mxfp4", x_scale=E_), S.E_ARG),
])
def test_linear_refuses(kw, status):
    assert _linear(**kw) == status and sp.spconv_last_error()


@pytest.mark.parametrize("kw", [dict(n=0), dict(cout=0), dict(n=0, x=None, w=None, y=None, ws=None)])
def test_linear_of_nothing(kw):
    assert _linear(**kw) == S.OK


def test_linear_workspace():
    size = sp.spconv_linear_mxfp4_workspace
    assert size("mxfp4", 1000, 4096, 4096) == 0
    assert size("bf16", 1000, 300, 64) == 1000 * 256 + 1000 * 2 * 8
    assert size("f32", 0, 300, 64) == 0
    with pytest.raises(sp.SpconvError):
        size("bf16", 10, 0, 64)
    with pytest.raises(sp.SpconvError):
        size("fp8", 10, 300, 64)
    assert S.load_library().spconv_linear_mxfp4_workspace(0, 1, 1, 1, None) == S.E_ARG


def _sample(**kw):
    a = dict(logits=A, dtype="f32", ld=500, u=B, n=4, vocab=500, temperatures=C, top_ks=D, top_ps=E_, min_ps=F,
             temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, ids=G, workspace=H, size=1 << 40)
    a.update(kw)
    return sp.spconv_sample(*a.values(), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), S.E_ARG), (dict(u=None), S.E_ARG), (dict(ids=None), S.E_ARG), (dict(n=-1), S.E_ARG),
    (dict(vocab=0), S.E_ARG), (dict(dtype="fp8"), S.E_ARG), (dict(ld=499), S.E_ARG),
    (dict(vocab=(1 << 20) + 1, ld=1 << 21), S.E_UNSUPPORTED), (dict(n=1 << 20), S.E_SHAPE), (dict(ld=1 << 40), S.E_SHAPE),
    (dict(temperatures=None, temperature=-0.5), S.E_ARG), (dict(temperatures=None, temperature=NAN), S.E_ARG),
    (dict(top_ks=None, top_k=-1), S.E_ARG), (dict(top_ps=None, top_p=1.5), S.E_ARG),
    (dict(top_ps=None, top_p=-0.1), S.E_ARG), (dict(top_ps=None, top_p=NAN), S.E_ARG),
    (dict(min_ps=None, min_p=1.5), S.E_ARG), (dict(min_ps=None, min_p=-0.1), S.E_ARG),
    (dict(min_ps=None, min_p=NAN), S.E_ARG), (dict(logits=A + 2), S.E_ARG), (dict(u=B + 2), S.E_ARG),
    (dict(temperatures=C + 1), S.E_ARG), (dict(top_ks=D + 1), S.E_ARG), (dict(top_ps=E_ + 1), S.E_ARG),
    (dict(min_ps=F + 1), S.E_ARG), (dict(ids=G + 2), S.E_ARG), (dict(workspace=H + 8), S.E_ARG),
    (dict(ids=A + 100), S.E_ARG), (dict(ids=B + 4), S.E_ARG), (dict(ids=D), S.E_ARG), (dict(ids=F + 12), S.E_ARG),
])
def test_sample_refuses(kw, status):
    assert _sample(**kw) == status and sp.spconv_last_error()


def test_sample_of_nothing():
    assert _sample(n=0, logits=None, u=None, ids=None, workspace=None, size=0) == S.OK


def test_sample_workspace():
    size = sp.spconv_sample_workspace
    for dtype in ("f32", "f16", "bf16"):
        assert size(dtype, 0, 500) == 0
        sizes = [size(dtype, n, 1 << 20) for n in (1, 7, 64)]
        assert sizes == sorted(sizes)
    with pytest.raises(sp.SpconvError):
        size("f32", 1, (1 << 20) + 1)
    assert S.load_library().spconv_sample_workspace(0, 1, 1, None) == S.E_ARG


def test_python_wrappers_refuse_host_tensors_and_wrong_shapes():
    import torch
    x = torch.zeros(4, 256)
    w = torch.zeros(4, 128, dtype=torch.uint8)
    for call in (lambda: sp.rms_norm(x), lambda: sp.rms_norm_fp8(x), lambda: sp.quantize_mxfp4(x),
                 lambda: sp.sample(x, torch.zeros(4)), lambda: sp.rms_norm(x[0]), lambda: sp.rms_norm(x.long()),
                 lambda: sp.quantize_mxfp4(x.long()), lambda: sp.sample(x.double(), torch.zeros(4)),
                 lambda: sp.Mxfp4Linear(w, torch.zeros(1, 4, 8, dtype=torch.uint8), 4, 256),
                 lambda: sp.Mxfp4Linear(w, torch.zeros(1, 4, 8, dtype=torch.uint8), 4, 256, act="gelu")):
        with pytest.raises(ValueError):
            call()


def test_mxfp4_is_no_plan_storage():
    status, plan = sp.spconv_plan_create(4, 4, 1, np.zeros(5, np.int32), np.zeros(1, np.int32),
                                         np.zeros(1, np.float32), storage=S.MXFP4, check=False)
    assert status == S.E_ARG and not plan


def test_library_takes_the_declared_arguments():
    """Every argument of the binding is one of the header's (name and count)."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "spconv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    lib = S.load_library()
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float,
             "spconv_dtype": ctypes.c_int32, "spconv_act": ctypes.c_int32}
    for name in ("spconv_rms_norm", "spconv_quantize_mxfp4", "spconv_linear_mxfp4", "spconv_linear_mxfp4_workspace",
                 "spconv_sample", "spconv_sample_workspace"):
        args = re.search(name + r"\(([^)]*)\)", text).group(1).split(",")
        declared = getattr(lib, name).argtypes
        assert len(args) == len(declared), name
        for arg, kind in zip(args, declared):
            if "*" in arg:
                assert kind is ctypes.c_void_p or issubclass(kind, ctypes._Pointer), (name, arg)
            else:
                assert kind is kinds[arg.split()[0]], (name, arg)


# ---- the references that the GPU tests compare with ----

def test_codes_of_the_borders():
    """Halfway goes to the even code, as the form's definition in bits has it."""
    v = np.array([0, 0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.0001, 6.99, -0.25, -0.75, -6.9, -0.0])
    assert e2m1(v).tolist() == [0, 0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 8, 10, 15, 8]


def test_powers_of_blocks():
    x = np.zeros((1, 320))
    x[0, 0], x[0, 32], x[0, 64], x[0, 96], x[0, 128] = 6.99, 7.0, -4.0, 3.99, 3.5
    x[0, 160], x[0, 192], x[0, 224], x[0, 256] = np.inf, np.nan, 2.0 ** -149, 3.4e38
    code, scale = quantize4_ref(x)
    assert scale[0].tolist() == [127, 128, 127, 127, 127, 255, 255, 0, 253] + [0] * 7
    q, s = packed(code, scale)
    back = unpacked(q, s)
    assert np.array_equal(back[0], code) and np.array_equal(back[1], scale)
    v = values4(code, scale, 320)[0]
    assert v[0] == 6 and v[32] == 8 and v[64] == -4 and v[96] == 4 and np.isnan(v[160:224]).all() and v[256] == 2.0 ** 128


def test_sampling_reference_by_hand():
    l = np.log(np.array([[0.1, 0.4, 0.3, 0.2]]))
    assert sample_ref(l, [0.05])[0] == 0 and sample_ref(l, [0.15])[0] == 1 and sample_ref(l, [0.95])[0] == 3
    assert sample_ref(l, [0.05], top_k=2)[0] == 1 and sample_ref(l, [0.6], top_k=2)[0] == 2
    assert sample_ref(l, [0.9], top_p=0.6)[0] == 2 and sample_ref(l, [0.9], top_p=0.3)[0] == 1
    assert sample_ref(l, [0.99], min_p=0.6)[0] == 2 and sample_ref(l, [0.99], temperature=0)[0] == 1
    assert sample_ref(np.full((1, 3), -np.inf), [0.5])[0] == -1
