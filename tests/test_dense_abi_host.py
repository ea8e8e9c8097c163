"""Refusals of the dense layers and of the AdamW step that need no GPU: every argument is checked before any work is enqueued."""
import ctypes as C

import pytest

import paper_2003_10735_amd as st

P = 4096            # a pointer that is never followed: validation comes first
F32, BF16 = st.ST_F32, st.ST_BF16


def mat(rows, cols, rs=None, cs=1, dtype=F32, data=P):
    return st.StMatrix(data, dtype, rows, cols, cols if rs is None else rs, cs)


def quantize(x=None, q=P, pitch=16, scale=P, ws=P):
    return st.lib().st_int8_quantize(C.byref(x) if x is not None else None, q, pitch, scale, ws, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), st.ST_ERR_NULL),
    (dict(x=mat(4, 0)), st.ST_ERR_SHAPE), (dict(x=mat(-1, 4)), st.ST_ERR_SHAPE), (dict(x=mat(1 << 31, 4)), st.ST_ERR_SHAPE), (dict(x=mat(1 << 24, 4)), st.ST_ERR_SHAPE),
    (dict(x=mat(4, 4, dtype=7)), st.ST_ERR_ARG), (dict(x=mat(4, 4, data=P + 2)), st.ST_ERR_ARG), (dict(x=mat(4, 4, data=None)), st.ST_ERR_NULL),
    (dict(x=mat(4, 4, rs=2, cs=8)), st.ST_ERR_SHAPE), (dict(x=mat(4, 4, rs=-4)), st.ST_ERR_SHAPE),
    (dict(x=mat(4, 17)), st.ST_ERR_SHAPE),                        # pitch below the row
    (dict(x=mat(4, 4), pitch=24), st.ST_ERR_SHAPE), (dict(x=mat(4, 4), pitch=(1 << 23) + 16), st.ST_ERR_SHAPE),
    (dict(x=mat(4, 4), q=None), st.ST_ERR_NULL), (dict(x=mat(4, 4), scale=None), st.ST_ERR_NULL),
    (dict(x=mat(4, 4), q=P + 8), st.ST_ERR_ARG), (dict(x=mat(4, 4), scale=P + 1), st.ST_ERR_ARG),
    (dict(x=mat(4, 4, rs=1, cs=4), ws=None), st.ST_ERR_WORKSPACE), (dict(x=mat(4, 4, rs=1, cs=4), ws=P + 128), st.ST_ERR_WORKSPACE),
    (dict(x=mat(0, 4)), st.ST_OK),
])
def test_quantize_refuses(kw, status):
    assert quantize(**kw) == status


def linear(x=None, wq=P, w_pitch=16, ws=P, n=8, bias=None, relu=0, y=P, dtype=F32, y_pitch=8, work=P):
    return st.lib().st_int8_linear(C.byref(x) if x is not None else None, wq, w_pitch, ws, n, bias, relu, y, dtype, y_pitch, work, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), st.ST_ERR_NULL), (dict(x=mat(3, 16), n=0), st.ST_ERR_SHAPE), (dict(x=mat(3, 0)), st.ST_ERR_SHAPE),
    (dict(x=mat(3, st.ST_INT8_MAX_SUM + 1), w_pitch=1 << 20), st.ST_ERR_SHAPE),
    (dict(x=mat(3, 17)), st.ST_ERR_SHAPE), (dict(x=mat(3, 16), w_pitch=20), st.ST_ERR_SHAPE), (dict(x=mat(3, 16), y_pitch=7), st.ST_ERR_SHAPE),
    (dict(x=mat(3, 16, rs=40, cs=2)), st.ST_ERR_SHAPE),
    (dict(x=mat(3, 16), dtype=2), st.ST_ERR_ARG), (dict(x=mat(3, 16), relu=2), st.ST_ERR_ARG), (dict(x=mat(3, 16), wq=P + 4), st.ST_ERR_ARG),
    (dict(x=mat(3, 16), bias=P + 2), st.ST_ERR_ARG), (dict(x=mat(3, 16), y=P + 2), st.ST_ERR_ARG),
    (dict(x=mat(3, 16), wq=None), st.ST_ERR_NULL), (dict(x=mat(3, 16), ws=None), st.ST_ERR_NULL), (dict(x=mat(3, 16), y=None), st.ST_ERR_NULL),
    (dict(x=mat(3, 16), work=None), st.ST_ERR_WORKSPACE), (dict(x=mat(3, 16), work=P + 16), st.ST_ERR_WORKSPACE),
    (dict(x=mat(0, 16), work=None), st.ST_OK),
])
def test_linear_refuses(kw, status):
    assert linear(**kw) == status


def backward(x=None, w=None, dy=None, y=None, dx=None, dxt=F32, dxp=16, dw=None, dwp=16, db=None, work=P):
    ref = [None if a is None else C.byref(a) for a in (x, w, dy, y)]
    return st.lib().st_int8_linear_backward(*ref, dx, dxt, dxp, dw, dwp, db, work, None)


@pytest.mark.parametrize("kw,status", [
    (dict(), st.ST_ERR_NULL), (dict(dy=mat(3, 8), dx=P), st.ST_ERR_NULL), (dict(dy=mat(3, 8), dw=P), st.ST_ERR_NULL),
    (dict(dy=mat(3, 8), w=mat(9, 16), dx=P), st.ST_ERR_SHAPE), (dict(dy=mat(3, 8), x=mat(4, 16), dw=P), st.ST_ERR_SHAPE),
    (dict(dy=mat(3, 0), db=P), st.ST_ERR_SHAPE), (dict(dy=mat(3, 8), w=mat(8, 16), dx=P, dxp=15), st.ST_ERR_SHAPE),
    (dict(dy=mat(3, 8), x=mat(3, 16), dw=P, dwp=15), st.ST_ERR_SHAPE),
    (dict(dy=mat(3, st.ST_INT8_MAX_SUM + 1), w=mat(st.ST_INT8_MAX_SUM + 1, 4), dx=P), st.ST_ERR_SHAPE),
    (dict(dy=mat((1 << 23) + 1, 1), x=mat((1 << 23) + 1, 1), dw=P), st.ST_ERR_SHAPE),
    (dict(dy=mat(3, 8), y=mat(3, 8, rs=1, cs=3), db=P), st.ST_ERR_SHAPE), (dict(dy=mat(3, 8), y=mat(3, 9), db=P), st.ST_ERR_SHAPE),
    (dict(dy=mat(3, 8), w=mat(8, 16), dx=P, dxt=5), st.ST_ERR_ARG), (dict(dy=mat(3, 8), db=P + 2), st.ST_ERR_ARG),
    (dict(dy=mat(3, 8), db=P, work=None), st.ST_ERR_WORKSPACE), (dict(dy=mat(3, 8), db=P, work=P + 4), st.ST_ERR_WORKSPACE),
])
def test_backward_refuses(kw, status):
    assert backward(**kw) == status


def tensor(n=10, decay=0.0, **kw):
    fields = dict(param=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, copy=None)
    fields.update(kw)
    return st.StAdamwTensor(*fields.values(), n, decay)


def step(tensors=None, count=None, ws=P, opts=True, **kw):
    o = dict(param_dtype=F32, grad_dtype=F32, state_bits=32, t=1, lr=0.1, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, max_norm=1.0,
             grad_norm=None)
    o.update(kw)
    tensors = [tensor()] if tensors is None else tensors
    a = (st.StAdamwTensor * max(1, len(tensors)))(*tensors)
    return st.lib().st_adamw_step(a, len(tensors) if count is None else count, C.byref(st.StAdamwOpts(*o.values())) if opts else None, ws, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,status", [
    (dict(opts=False), st.ST_ERR_NULL), (dict(count=-1), st.ST_ERR_SHAPE), (dict(count=65537), st.ST_ERR_SHAPE),
    (dict(tensors=[tensor(n=-1)]), st.ST_ERR_SHAPE), (dict(tensors=[tensor(n=(1 << 33) + 1)]), st.ST_ERR_SHAPE),
    (dict(tensors=[tensor(decay=NAN)]), st.ST_ERR_ARG),
    *[(dict([(k, v)]), st.ST_ERR_ARG) for k, v in (
        ("param_dtype", 3), ("grad_dtype", -1), ("state_bits", 16), ("t", 0), ("lr", NAN), ("lr", INF), ("beta1", 1.0), ("beta1", -0.1),
        ("beta2", 1.0), ("beta2", NAN), ("eps", -1.0), ("eps", INF), ("grad_scale", 0.0), ("grad_scale", NAN), ("grad_scale", 1e-60),
        ("max_norm", -1.0), ("max_norm", INF), ("max_norm", 1e-60), ("grad_norm", P + 2))],
    *[(dict(tensors=[tensor(**{k: None})]), st.ST_ERR_NULL) for k in ("param", "grad", "m", "v")],
    *[(dict(tensors=[tensor(**{k: None})], state_bits=8), st.ST_ERR_NULL) for k in ("m_scale", "v_scale")],
    *[(dict(tensors=[tensor(**{k: P + 1})]), st.ST_ERR_ARG) for k in ("param", "grad", "m", "v", "copy")],
    (dict(tensors=[tensor(v_scale=P + 2)], state_bits=8), st.ST_ERR_ARG),
    (dict(ws=None), st.ST_ERR_WORKSPACE), (dict(ws=P + 8), st.ST_ERR_WORKSPACE), (dict(ws=None, max_norm=0.0, grad_norm=P), st.ST_ERR_WORKSPACE),
    (dict(tensors=[], ws=None, max_norm=0.0), st.ST_OK), (dict(tensors=[tensor(n=0, param=None)], ws=None, max_norm=0.0), st.ST_OK),
])
def test_adamw_refuses(kw, status):
    assert step(**kw) == status


def test_state_refuses():
    f = st.lib().st_adamw_state
    assert f(P, P, P, P, -1, P, P, None) == st.ST_ERR_SHAPE
    assert f(None, P, P, P, 5, P, P, None) == st.ST_ERR_NULL and f(P, P, P, None, 5, P, P, None) == st.ST_ERR_NULL
    assert f(P, P + 2, P, P, 5, P, P, None) == st.ST_ERR_ARG and f(P, P, P, P, 5, P + 1, P, None) == st.ST_ERR_ARG
    assert f(None, None, None, None, 0, None, None, None) == st.ST_OK and f(P, P, P, P, 5, None, None, None) == st.ST_OK


def test_workspace_sizes():
    L = st.lib()
    assert L.st_int8_linear_workspace(0, 1, 1) > 0 and L.st_int8_linear_workspace(1, 0, 1) == 0
    assert L.st_int8_linear_workspace(5, 7, st.ST_INT8_MAX_SUM + 1) == 0 and L.st_int8_linear_workspace(-1, 7, 3) == 0
    assert L.st_int8_linear_workspace(1000, 64, 256) >= 1000 * 256 + 4000
    assert L.st_int8_linear_backward_workspace(100, 64, 256) >= 100 * 128 + (64 + 256) * 128 + 256 * 128
    assert L.st_int8_linear_backward_workspace(100, 0, 256) == 0
    assert L.st_int8_quantize_workspace(10, 0) == 0 and L.st_int8_quantize_workspace(0, 4) > 0
    a = (st.StAdamwTensor * 2)(tensor(n=5), tensor(n=5000))
    assert L.st_adamw_workspace(a, 2) > 256 and L.st_adamw_workspace(a, -1) == 0


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    f, i8 = (lambda *s: torch.zeros(*s)), (lambda *s: torch.zeros(*s, dtype=torch.int8))
    with pytest.raises(st.StError):
        st.st_int8_linear(f(3, 16).half(), i8(8, 16), f(8))
    with pytest.raises(st.StError):
        st.st_int8_linear(f(2, 3, 16), i8(8, 16), f(8))
    with pytest.raises(st.StError):
        st.st_int8_linear(f(3, 16), i8(8, 16), f(7))
    with pytest.raises(st.StError):
        st.st_int8_linear(f(3, 16), i8(8, 8), f(8))
    with pytest.raises(st.StError):
        st.st_int8_linear(f(3, 16), i8(8, 16), f(8), out=f(3, 9))
    with pytest.raises(st.StError):
        st.st_int8_linear_backward(f(3, 16), f(8, 16), f(3, 8), dw=f(8, 16).bfloat16())
    with pytest.raises(st.StError):
        st.AdamWTensors([f(4)], [f(5)], [f(4)], [f(4)])
    with pytest.raises(st.StError):
        st.AdamWTensors([f(4)], [f(4)], [i8(4)], [i8(4).to(torch.uint8)])
    with pytest.raises(st.StError):
        st.AdamWTensors([f(4, 4).t()], [f(16)], [f(16)], [f(16)])
    with pytest.raises(st.StError):
        st.new_adamw_state([f(4)], bits=4)
    t = st.AdamWTensors([f(4)], [f(4)], [f(4)], [f(4)])
    with pytest.raises(st.StError):
        t.set_grads([f(5)])
