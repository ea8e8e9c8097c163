"""Refusals of the dense layers in bfloat16 and float32 and of the clipping of gradients that need no GPU: every argument is checked before any
work is enqueued; and what their binding checks and makes before it calls the library."""
import ctypes as C

import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")

P = 4096            # a pointer that is never followed: validation comes first
F32, BF16 = st.ST_F32, st.ST_BF16
BIG = 1 << 40


def mat(rows, cols, rs=None, cs=1, dtype=F32, data=P):
    return st.StMatrix(data, dtype, rows, cols, cols if rs is None else rs, cs)


def ref(a):
    return None if a is None else C.byref(a)


def linear(x=mat(3, 16), w=mat(8, 16), opts=None, y=P, dtype=F32, pitch=8, ws=P, nbytes=BIG):
    return st.lib().st_linear(ref(x), ref(w), None if opts is None else C.byref(st.StLinearOpts(**opts)), y, dtype, pitch, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), st.ST_ERR_NULL), (dict(w=None), st.ST_ERR_NULL), (dict(y=None), st.ST_ERR_NULL),
    (dict(x=mat(3, 16, data=None)), st.ST_ERR_NULL), (dict(w=mat(8, 16, data=None)), st.ST_ERR_NULL),
    (dict(x=mat(3, 0), w=mat(8, 0)), st.ST_ERR_SHAPE), (dict(w=mat(0, 16)), st.ST_ERR_SHAPE), (dict(x=mat(-1, 16)), st.ST_ERR_SHAPE),
    (dict(w=mat(8, 17)), st.ST_ERR_SHAPE), (dict(x=mat(1 << 24, 16)), st.ST_ERR_SHAPE),
    (dict(x=mat(3, st.ST_LINEAR_MAX_CHANNELS + 1), w=mat(8, st.ST_LINEAR_MAX_CHANNELS + 1)), st.ST_ERR_SHAPE),
    (dict(w=mat(st.ST_LINEAR_MAX_CHANNELS + 1, 16), pitch=1 << 22), st.ST_ERR_SHAPE),
    (dict(x=mat(3, 16, rs=40, cs=2)), st.ST_ERR_SHAPE), (dict(w=mat(8, 16, rs=-16)), st.ST_ERR_SHAPE), (dict(w=mat(8, 16, rs=(1 << 40) + 1)), st.ST_ERR_SHAPE),
    (dict(pitch=7), st.ST_ERR_SHAPE), (dict(opts=dict(residual=P, residual_pitch=7)), st.ST_ERR_SHAPE), (dict(opts=dict(pre=P, pre_pitch=7)), st.ST_ERR_SHAPE),
    (dict(x=mat(3, 16, dtype=2), w=mat(8, 16, dtype=2)), st.ST_ERR_ARG), (dict(x=mat(3, 16, dtype=BF16)), st.ST_ERR_ARG), (dict(w=mat(8, 16, dtype=BF16)), st.ST_ERR_ARG),
    (dict(dtype=2), st.ST_ERR_ARG), (dict(opts=dict(activation=5)), st.ST_ERR_ARG), (dict(opts=dict(activation=-1)), st.ST_ERR_ARG),
    (dict(opts=dict(residual=P, residual_pitch=8, residual_dtype=3)), st.ST_ERR_ARG), (dict(opts=dict(pre=P, pre_pitch=8, pre_dtype=-1)), st.ST_ERR_ARG),
    (dict(x=mat(3, 16, data=P + 2)), st.ST_ERR_ARG), (dict(w=mat(8, 16, data=P + 1)), st.ST_ERR_ARG), (dict(y=P + 2), st.ST_ERR_ARG), (dict(y=P + 1, dtype=BF16), st.ST_ERR_ARG),
    (dict(opts=dict(bias=P + 2)), st.ST_ERR_ARG), (dict(opts=dict(residual=P + 2, residual_pitch=8)), st.ST_ERR_ARG), (dict(opts=dict(pre=P + 2, pre_pitch=8)), st.ST_ERR_ARG),
    (dict(opts=dict(residual=P, residual_pitch=9)), st.ST_ERR_ARG), (dict(opts=dict(residual=P, residual_pitch=8, residual_dtype=BF16)), st.ST_ERR_ARG),
    # rows of three floats behind one another have to be copied, tiles of two products in parts have to be kept
    (dict(x=mat(3000, 3), w=mat(3000, 3), pitch=3000, ws=None), st.ST_ERR_WORKSPACE), (dict(x=mat(3000, 3), w=mat(3000, 3), pitch=3000, nbytes=100), st.ST_ERR_WORKSPACE),
    (dict(x=mat(3000, 3), w=mat(3000, 3), pitch=3000, ws=P + 64), st.ST_ERR_WORKSPACE),
    (dict(x=mat(0, 16), y=None, ws=None, nbytes=0), st.ST_OK),
])
def test_linear_refuses(kw, status):
    assert linear(**kw) == status


def backward(x=mat(3, 16), w=mat(8, 16), dy=mat(3, 8), pre=None, act=0, ws=P, nbytes=BIG, grads=True, **g):
    fields = dict(dx=P, dx_pitch=16, dx_dtype=F32, dw=P, dw_pitch=16, dw_dtype=F32, db=P)
    fields.update(g)
    return st.lib().st_linear_backward(ref(x), ref(w), ref(dy), ref(pre), act, C.byref(st.StLinearGrads(**fields)) if grads else None, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(grads=False), st.ST_ERR_NULL), (dict(dy=None), st.ST_ERR_NULL), (dict(x=None), st.ST_ERR_NULL), (dict(w=None), st.ST_ERR_NULL),
    (dict(act=2), st.ST_ERR_NULL), (dict(act=2, pre=mat(3, 8, data=None)), st.ST_ERR_NULL),
    (dict(w=mat(9, 16)), st.ST_ERR_SHAPE), (dict(x=mat(4, 16)), st.ST_ERR_SHAPE), (dict(x=mat(3, 15)), st.ST_ERR_SHAPE), (dict(dy=mat(3, 0)), st.ST_ERR_SHAPE),
    (dict(act=2, pre=mat(3, 9)), st.ST_ERR_SHAPE), (dict(dx_pitch=15), st.ST_ERR_SHAPE), (dict(dw_pitch=15), st.ST_ERR_SHAPE),
    (dict(dy=mat(3, 8, rs=20, cs=2)), st.ST_ERR_SHAPE), (dict(dy=mat(1 << 24, 8), x=mat(1 << 24, 16)), st.ST_ERR_SHAPE),
    (dict(act=5, pre=mat(3, 8)), st.ST_ERR_ARG), (dict(x=mat(3, 16, dtype=BF16)), st.ST_ERR_ARG), (dict(dx_dtype=2), st.ST_ERR_ARG), (dict(dw_dtype=-1), st.ST_ERR_ARG),
    (dict(accumulate=2), st.ST_ERR_ARG), (dict(dx=P + 2), st.ST_ERR_ARG), (dict(dw=P + 1), st.ST_ERR_ARG), (dict(db=P + 2), st.ST_ERR_ARG), (dict(dy=mat(3, 8, data=P + 2)), st.ST_ERR_ARG),
    (dict(ws=None), st.ST_ERR_WORKSPACE), (dict(ws=P + 8), st.ST_ERR_WORKSPACE), (dict(nbytes=0), st.ST_ERR_WORKSPACE),
    (dict(dx=None, dw=None, db=None, ws=None, nbytes=0), st.ST_OK),
    (dict(dy=mat(0, 8), x=mat(0, 16), accumulate=1, ws=None, nbytes=0), st.ST_OK),
])
def test_backward_refuses(kw, status):
    assert backward(**kw) == status


def test_workspace_sizes():
    L = st.lib()
    size = lambda x, w: L.st_linear_workspace(ref(x), ref(w))      # noqa: E731
    assert size(mat(4096, 4096, dtype=BF16), mat(4096, 4096, dtype=BF16)) == 256         # nothing to copy, nothing to join
    assert size(mat(1, 1003, dtype=BF16), mat(5000, 1003, dtype=BF16)) == 256            # few tokens: at any address
    assert size(mat(4096, 1003, dtype=BF16), mat(4096, 1003, dtype=BF16)) >= 2 * 4096 * 1003 * 2
    assert size(mat(0, 4), mat(4, 4)) == 256 and size(None, mat(4, 4)) == 0 and size(mat(4, 4), mat(4, 5)) == 0
    back = lambda x, w, dy, act=0: L.st_linear_backward_workspace(ref(x), ref(w), ref(dy), act)      # noqa: E731
    assert back(mat(64, 32), mat(16, 32), mat(64, 16), 2) >= 64 * 16 * 4                  # dz
    assert back(None, None, mat(64, 16)) >= 256 + 16 * 4 and back(mat(4, 4), mat(4, 4), None) == 0 and back(mat(4, 4), mat(4, 4), mat(4, 4), 9) == 0


def tensor(n=10, grad=P, out=P, gd=F32, od=F32):
    return st.StGradTensor(grad, out, n, gd, od)


def clip(tensors=None, count=None, scale=1.0, max_norm=1.0, norm=None, ws=P):
    tensors = [tensor()] if tensors is None else tensors
    a = (st.StGradTensor * max(1, len(tensors)))(*tensors)
    return st.lib().st_grad_clip(a, len(tensors) if count is None else count, scale, max_norm, norm, ws, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,status", [
    (dict(count=-1), st.ST_ERR_SHAPE), (dict(count=65537), st.ST_ERR_SHAPE), (dict(tensors=[tensor(n=-1)]), st.ST_ERR_SHAPE),
    (dict(tensors=[tensor(n=(1 << 33) + 1)]), st.ST_ERR_SHAPE), (dict(tensors=[tensor(n=1 << 33), tensor(n=1)]), st.ST_ERR_SHAPE),
    (dict(tensors=[tensor(grad=None)]), st.ST_ERR_NULL), (dict(tensors=[tensor(), tensor(out=None)]), st.ST_ERR_NULL),
    (dict(tensors=[tensor(gd=2)]), st.ST_ERR_ARG), (dict(tensors=[tensor(od=-1)]), st.ST_ERR_ARG), (dict(tensors=[tensor(grad=P + 2, out=P + 2)]), st.ST_ERR_ARG),
    (dict(tensors=[tensor(out=P + 1001)]), st.ST_ERR_ARG),
    (dict(tensors=[tensor(od=BF16)]), st.ST_ERR_ARG), (dict(tensors=[tensor(out=P + 4)]), st.ST_ERR_ARG), (dict(tensors=[tensor(out=P - 36)]), st.ST_ERR_ARG),
    *[(dict([(k, v)]), st.ST_ERR_ARG) for k, v in (("scale", 0.0), ("scale", -1.0), ("scale", NAN), ("scale", INF), ("scale", 1e-60), ("max_norm", -1.0), ("max_norm", NAN),
                                                 ("max_norm", INF), ("max_norm", 1e-60), ("norm", P + 2))],
    (dict(ws=None), st.ST_ERR_WORKSPACE), (dict(ws=P + 8), st.ST_ERR_WORKSPACE),
    (dict(tensors=[], ws=None), st.ST_OK), (dict(tensors=[tensor(n=0, grad=None, out=None)], ws=None), st.ST_OK), (dict(tensors=[tensor(out=None)], ws=None), st.ST_OK),
])
def test_clip_refuses(kw, status):
    assert clip(**kw) == status


# ---------------------------------------------------------------------------------------------------------------- the binding
class OnDevice(torch.Tensor):
    is_cuda = True


class Recorder:
    """The library, with entry points that only note how they were called."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name not in ("st_linear", "st_linear_backward", "st_grad_clip"):
            return getattr(self.real, name)

        def entry(*args):
            self.calls.append((name, args))
            return st.ST_OK
        return entry


@pytest.fixture
def library(monkeypatch):
    recorder, empty = Recorder(st.lib()), torch.empty
    monkeypatch.setattr(st, "_LIB", recorder)
    monkeypatch.setattr(st, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(OnDevice))
    return recorder


def dev(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


B = torch.bfloat16


@pytest.mark.parametrize("status,call", [
    (st.ST_ERR_NULL, lambda: st.st_linear(None, dev(8, 16))), (st.ST_ERR_NULL, lambda: st.st_linear(dev(3, 16), None)),
    (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(2, 3, 16), dev(8, 16))), (st.ST_ERR_ARG, lambda: st.st_linear(dev(3, 16).half(), dev(8, 16))),
    (st.ST_ERR_ARG, lambda: st.st_linear(torch.zeros(3, 16), dev(8, 16))), (st.ST_ERR_ARG, lambda: st.st_linear(dev(3, 16), torch.zeros(8, 16))),
    (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(3, 16), dev(8, 16), bias=dev(7))), (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(3, 16), dev(8, 16), bias=dev(8, dtype=B))),
    (st.ST_ERR_ARG, lambda: st.st_linear(dev(3, 16), dev(8, 16), bias=torch.zeros(8))),
    (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(3, 16), dev(8, 16), residual=dev(3, 9))), (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(3, 16), dev(8, 16), residual=dev(8, 3).t())),
    (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(3, 16), dev(8, 16), pre=dev(4, 8))), (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(3, 16), dev(8, 16), out=dev(3, 9))),
    (st.ST_ERR_ARG, lambda: st.st_linear(dev(3, 16), dev(8, 16), out=torch.zeros(3, 8))), (st.ST_ERR_WORKSPACE, lambda: st.st_linear(dev(3, 16), dev(8, 16), workspace=torch.zeros(512, dtype=torch.uint8))),
    (st.ST_ERR_SHAPE, lambda: st.st_linear(dev(3, 16), dev(8, 17))), (st.ST_ERR_SHAPE, lambda: st.new_linear_workspace(dev(3, 16), dev(8, 17))),
    (st.ST_ERR_NULL, lambda: st.new_linear_workspace(dev(3, 16), None)), (st.ST_ERR_NULL, lambda: st.new_linear_workspace(None, None, None)),
    (st.ST_ERR_NULL, lambda: st.st_linear_backward(None, dev(8, 16), dev(3, 8), dw=dev(8, 16))), (st.ST_ERR_NULL, lambda: st.st_linear_backward(dev(3, 16), None, dev(3, 8), dx=dev(3, 16))),
    (st.ST_ERR_NULL, lambda: st.st_linear_backward(dev(3, 16), None, dev(3, 8), None, st.ST_ACT_SILU, dw=dev(8, 16))),
    (st.ST_ERR_SHAPE, lambda: st.st_linear_backward(dev(3, 16), None, dev(3, 8), dw=dev(9, 16))), (st.ST_ERR_SHAPE, lambda: st.st_linear_backward(None, dev(8, 16), dev(3, 8), dx=dev(16, 3).t())),
    (st.ST_ERR_SHAPE, lambda: st.st_linear_backward(None, None, dev(3, 8), db=dev(9))), (st.ST_ERR_ARG, lambda: st.st_linear_backward(None, None, torch.zeros(3, 8), db=dev(8))),
    (st.ST_ERR_SHAPE, lambda: st.GradTensors([dev(4)], [dev(5)])), (st.ST_ERR_SHAPE, lambda: st.GradTensors([dev(4)], [])), (st.ST_ERR_NULL, lambda: st.GradTensors([None])),
    (st.ST_ERR_SHAPE, lambda: st.GradTensors([dev(4, 4).t()])), (st.ST_ERR_ARG, lambda: st.GradTensors([dev(4).half()])),
    (st.ST_ERR_ARG, lambda: st.st_grad_clip(st.GradTensors([torch.zeros(4)]))),
    (st.ST_ERR_WORKSPACE, lambda: st.st_grad_clip(st.GradTensors([dev(4)]), 1.0, workspace=dev(8, dtype=torch.uint8))),
    (st.ST_ERR_SHAPE, lambda: st.st_grad_clip(st.GradTensors([dev(4)]), 1.0, grad_norm=dev(2))),
])
def test_binding_refuses(status, call, library):
    with pytest.raises(st.StError) as e:
        call()
    assert e.value.status == status and not library.calls


def test_lists_whose_tensors_overlap_are_refused():
    a, b = dev(20), dev(20)
    h = dev(20, dtype=B)
    for grads, outs in (([a, a], None), ([a[:12], a[8:]], None), ([a, b], [b, a]), ([a[:10], b[:10]], [b[10:], b[10:]]),
                        ([a[:10]], [a[5:15]]), ([h[:10], a[:10]], [a[5:15], b[:10]])):
        with pytest.raises(st.StError) as e:
            st.GradTensors(grads, outs)
        assert e.value.status == st.ST_ERR_ARG
    st.GradTensors([a[:10], a[10:], h], [b[:10], a[10:], dev(20)])       # apart, in place, and apart in another type
    st.GradTensors([a, a[:0], a[:0]])                                    # nothing is nobody's
    st.GradTensors([a, a], [b, dev(20)])                                 # read twice, written apart


def test_calls_that_get_through(library):
    st.st_linear(dev(3, 16, dtype=B), dev(8, 16, dtype=B), dev(8), st.ST_ACT_GELU, residual=dev(3, 8), pre=dev(3, 8, dtype=B), out_dtype=torch.float32)
    st.st_linear_backward(dev(3, 16), dev(8, 16), dev(8, 3).t(), dev(3, 8, dtype=B), st.ST_ACT_GELU, dx=dev(3, 16), dw=dev(8, 16, dtype=B), db=dev(8), accumulate=True)
    st.st_grad_clip(st.GradTensors([dev(4), dev(5, dtype=B)]), 1.0, 0.5, dev(1))
    (a, x), (b, y), (c, z) = library.calls
    assert (a, b, c) == ("st_linear", "st_linear_backward", "st_grad_clip") and x[4:6] == (st.ST_F32, 8) and y[4] == st.ST_ACT_GELU and z[1:4] == (2, 0.5, 1.0)


def test_structs_as_bytes_are_the_structs():
    """What the binding packs in one go lies as the ctypes structures do."""
    for packed, values, cls in ((st._MATRIX_BYTES, (P, 1, 3, 16, 40, 1), st.StMatrix), (st._OPTS_BYTES, (P, 2, 1, P + 8, 9, P + 16, 10, 1), st.StLinearOpts),
                                (st._GRADS_BYTES, (P, 16, 1, 1, P + 8, 17, P + 16, 1), st.StLinearGrads)):
        assert packed.size == C.sizeof(cls)
        got = cls.from_buffer_copy(packed.pack(*values))
        assert tuple(getattr(got, name) for name, _ in cls._fields_) == values
