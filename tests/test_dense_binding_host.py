"""What the binding of the dense layers and of the AdamW step checks and makes before it calls the library, without a GPU.

The tensors are host tensors that say they are on a device, and the entry points are stand-ins that record their arguments (other
functions, those that give sizes among them, are the library's own): a call that gets through reaches the stand-in and nothing else.
"""
import types

import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")


class OnDevice(torch.Tensor):
    is_cuda = True


ENTRY_POINTS = ("st_int8_quantize", "st_int8_linear", "st_int8_linear_backward", "st_adamw_step", "st_adamw_state",
                "st_head_forward", "st_partial_distill", "st_miou", "st_object_weights")


class Recorder:
    """The library, with entry points that only note how they were called."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name not in ENTRY_POINTS:
            return getattr(self.real, name)

        def entry(*args):
            self.calls.append((name, args))
            return st.ST_OK
        return entry


@pytest.fixture
def library(monkeypatch):
    recorder, empty = Recorder(st.lib()), torch.empty
    monkeypatch.setattr(st, "_LIB", recorder)
    monkeypatch.setattr(st, "_stream", lambda stream: 0 if stream is None else stream.cuda_stream)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(OnDevice))
    return recorder


def dev(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def refused(status, call, library):
    with pytest.raises(st.StError) as e:
        call()
    assert e.value.status == status and not library.calls


# (rows, cols, buffer's width, first and last column of the view): what is written has to lie inside the view
@pytest.mark.parametrize("rows,cols,width,first,end,fits", [
    (4, 240, 256, 0, 256, True), (4, 240, 256, 16, 256, False), (4, 240, 256, 0, 240, False), (4, 200, 208, 0, 208, True),
    (4, 200, 208, 0, 200, False), (4, 100, 512, 256, 384, True), (4, 100, 512, 256, 368, False), (4, 130, 512, 0, 256, True),
    (4, 130, 512, 368, 512, False), (4, 300, 512, 0, 16, False), (4, 128, 256, 128, 256, True), (4, 16, 48, 16, 48, False),
    (1, 200, 512, 0, 208, True), (1, 200, 512, 0, 192, False), (0, 200, 512, 0, 512, True),
])
@pytest.mark.parametrize("columns", [False, True])
def test_codes_are_written_inside_what_is_given(rows, cols, width, first, end, fits, columns, library):
    x = dev(cols, rows).t() if columns else dev(rows, cols)
    q = dev(rows, width, dtype=torch.int8)[:, first:end]

    def call():
        st.st_int8_quantize(x, q=q)

    if not fits:
        refused(st.ST_ERR_SHAPE, call, library)
        return
    call()
    (name, args), = library.calls
    pitch, written = args[2], min((cols + 127) // 128 * 128, args[2])
    assert name == "st_int8_quantize" and args[1] == q.data_ptr()
    assert pitch == (q.stride(0) if rows > 1 else q.shape[1]) and written <= q.shape[1]


class Streams:
    """Stands in for torch's current stream: which one every tensor was made on, and which others may use it."""

    def __init__(self, monkeypatch):
        self.current, self.made, empty = "current", [], torch.empty

        class Scope:
            def __init__(scope, stream):
                scope.stream = stream

            def __enter__(scope):
                scope.before, self.current = self.current, scope.stream

            def __exit__(scope, *e):
                self.current = scope.before

        def make(*a, **k):
            k.pop("device", None)
            t = empty(*a, **k).as_subclass(OnDevice)
            self.made.append([t.data_ptr(), self.current, None, t])
            return t

        def record(t, stream):
            next(m for m in self.made if m[0] == t.data_ptr())[2] = stream

        monkeypatch.setattr(torch, "empty", make)
        monkeypatch.setattr(torch.cuda, "stream", Scope)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("stream", handle))
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(OnDevice, "record_stream", record, raising=False)


SMALL = st.HeadDesc(1, 8, 4, 4, 8, 8, 3, compute=st.ST_COMPUTE_F32)
# a call without its workspace and its results, how many of each it makes, and the entry point
CALLS = {
    "quantize rows": (lambda s: st.st_int8_quantize(dev(5, 24), stream=s), 0, 2),
    "quantize columns": (lambda s: st.st_int8_quantize(dev(24, 5).t(), stream=s), 1, 2),
    "linear": (lambda s: st.st_int8_linear(dev(5, 16), dev(7, 16, dtype=torch.int8), dev(7), stream=s), 1, 1),
    "backward": (lambda s: st.st_int8_linear_backward(dev(5, 16), dev(7, 16), dev(5, 7), dw=dev(7, 16), stream=s), 1, 0),
    "adamw": (lambda s: st.st_adamw_step(st.AdamWTensors([dev(9)], [dev(9)], [dev(9)], [dev(9)]), 1, 0.1, max_norm=1.0, stream=s), 1, 0),
    "state": (lambda s: st.st_adamw_state(dev(9, dtype=torch.int8), dev(1), dev(9, dtype=torch.uint8), dev(1), stream=s), 0, 2),
    "head forward": (lambda s: st.st_head_forward(SMALL, dev(1), dev(1), stream=s), 1, 0),
    "distill": (lambda s: st.st_partial_distill(SMALL, dev(1), dev(1), dev(1), 1, 0.1, stream=s), 1, 0),
    "miou": (lambda s: st.st_miou(dev(4, dtype=torch.uint8), dev(4, dtype=torch.int32), 3, stream=s), 0, 2),
    "object weights": (lambda s: st.st_object_weights(dev(1, 4, 4, dtype=torch.int32), 3, 1, stream=s), 0, 1),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("given", [False, True])
def test_what_a_call_makes_belongs_to_its_stream(name, given, library, monkeypatch):
    """Scratch and results are made on the stream that the call works on; results may be used on the caller's stream too."""
    call, scratch, results = CALLS[name]
    streams = Streams(monkeypatch)
    call(types.SimpleNamespace(cuda_stream=77) if given else None)
    assert [args[-1] for _, args in library.calls] == [77 if given else 0]
    assert len(streams.made) == scratch + results
    for address, made_on, also_on, _ in streams.made:
        assert made_on == (("stream", 77) if given else "current")
    assert sum(also_on is not None for _, _, also_on, _ in streams.made) == (results if given else 0)
    assert all(also_on in (None, "current") for _, _, also_on, _ in streams.made)


BAD_GRADIENTS = {                                    # made from the length that is wanted
    "length": (lambda n: dev(n + 1), st.ST_ERR_SHAPE), "type": (lambda n: dev(n, dtype=torch.bfloat16), st.ST_ERR_SHAPE),
    "order": (lambda n: dev(n, 2)[:, 0], st.ST_ERR_SHAPE), "host": (lambda n: torch.zeros(n), st.ST_ERR_ARG),
}


@pytest.mark.parametrize("bad", BAD_GRADIENTS)
@pytest.mark.parametrize("at", [0, 1, 2])
def test_refused_gradients_change_nothing(bad, at, library):
    """Whichever tensor of the new list is refused: the list goes on with the gradients that it had, and keeps them."""
    make, status = BAD_GRADIENTS[bad]
    params, first, second, m, v = ([dev(4), dev(5), dev(7)] for _ in range(5))
    tensors = st.AdamWTensors(params, first, m, v)
    wrong = list(second)
    wrong[at] = make(params[at].numel())
    refused(status, lambda: tensors.set_grads(wrong), library)
    assert [a.grad for a in tensors.array] == [t.data_ptr() for t in first] and all(a is b for a, b in zip(tensors.kept[1], first))
    refused(st.ST_ERR_SHAPE, lambda: tensors.set_grads(second[:2]), library)
    assert [a.grad for a in tensors.array] == [t.data_ptr() for t in first]
    tensors.set_grads(second)
    assert [a.grad for a in tensors.array] == [t.data_ptr() for t in second] and all(a is b for a, b in zip(tensors.kept[1], second))


@pytest.mark.parametrize("dtype", [torch.uint8, torch.bool, torch.float8_e4m3fn, torch.int16, torch.float32])
def test_codes_of_another_type_are_refused(dtype, library):
    """Weights are int8, codes of m int8 and of v uint8, scales float32: no other type of the same size is read as one of them."""
    refused(st.ST_ERR_SHAPE, lambda: st.st_int8_linear(dev(5, 16), dev(7, 16, dtype=dtype), dev(7)), library)
    i8, u8 = dev(9, dtype=torch.int8), dev(9, dtype=torch.uint8)
    refused(st.ST_ERR_SHAPE, lambda: st.st_adamw_state(dev(9, dtype=dtype), dev(1), u8, dev(1)), library)
    if dtype != torch.uint8:
        refused(st.ST_ERR_SHAPE, lambda: st.st_adamw_state(i8, dev(1), dev(9, dtype=dtype), dev(1)), library)
    refused(st.ST_ERR_SHAPE, lambda: st.st_adamw_state(i8, dev(1), i8, dev(1)), library)
    for scales in ((dev(1, dtype=torch.int32), dev(1)), (dev(1), dev(1, dtype=torch.int32))):
        refused(st.ST_ERR_SHAPE, lambda: st.st_adamw_state(i8, scales[0], u8, scales[1]), library)
    st.st_int8_linear(dev(5, 16), dev(7, 16, dtype=torch.int8), dev(7))
    st.st_adamw_state(i8, dev(1), u8, dev(1))
    assert [name for name, _ in library.calls] == ["st_int8_linear", "st_adamw_state"]


I8 = dev(7, 16, dtype=torch.int8)
MISSING = {
    "quantize": lambda: st.st_int8_quantize(None), "tokens": lambda: st.st_int8_linear(None, I8, dev(7)),
    "weights": lambda: st.st_int8_linear(dev(5, 16), None, dev(7)), "scales": lambda: st.st_int8_linear(dev(5, 16), I8, None),
    "dy": lambda: st.st_int8_linear_backward(dev(5, 16), dev(7, 16), None, dw=dev(7, 16)),
    "dx without w": lambda: st.st_int8_linear_backward(dev(5, 16), None, dev(5, 7), dx=dev(5, 16)),
    "dw without x": lambda: st.st_int8_linear_backward(None, dev(7, 16), dev(5, 7), dw=dev(7, 16)),
    "dx without either": lambda: st.st_int8_linear_backward(None, None, dev(5, 7), dx=dev(5, 16)),
    "first gradient": lambda: st.AdamWTensors([dev(4)], [None], [dev(4)], [dev(4)]),
    "second state": lambda: st.AdamWTensors([dev(4), dev(5)], [dev(4), dev(5)], [dev(4), None], [dev(4), dev(5)]),
    "new gradient": lambda: st.AdamWTensors([dev(4)], [dev(4)], [dev(4)], [dev(4)]).set_grads([None]),
    "codes": lambda: st.st_adamw_state(None, None, dev(9, dtype=torch.uint8), dev(1)),
    "codes of v": lambda: st.st_adamw_state(dev(9, dtype=torch.int8), dev(1), None, None, v_out=dev(9)),
    "state's scales": lambda: st.st_adamw_state(dev(9, dtype=torch.int8), None, None, None, m_out=dev(9)),
}
DIMENSIONS = {
    "quantize": lambda: st.st_int8_quantize(dev(16)), "tokens": lambda: st.st_int8_linear(dev(2, 3, 16), I8, dev(7)),
    "weights": lambda: st.st_int8_linear(dev(5, 16), dev(112, dtype=torch.int8), dev(7)),
    "dy": lambda: st.st_int8_linear_backward(dev(5, 16), None, dev(1, 5, 7), dw=dev(7, 16)),
    "dy of one": lambda: st.st_int8_linear_backward(dev(5, 16), None, dev(7), dw=dev(7, 16)),
    "x": lambda: st.st_int8_linear_backward(dev(5, 4, 4), None, dev(5, 7), dw=dev(7, 16)),
    "w": lambda: st.st_int8_linear_backward(None, dev(7), dev(5, 7), dx=dev(5, 16)),
    "y": lambda: st.st_int8_linear_backward(None, None, dev(5, 7), y=dev(35), db=dev(7)),
}


@pytest.mark.parametrize("name", MISSING)
def test_missing_tensors_are_the_librarys_error(name, library):
    refused(st.ST_ERR_NULL, MISSING[name], library)


@pytest.mark.parametrize("name", DIMENSIONS)
def test_matrices_have_two_dimensions(name, library):
    refused(st.ST_ERR_SHAPE, DIMENSIONS[name], library)


# Each call is right but for one argument.  name: (call with replacements, the entry point, {what is replaced: (by what, status)})
def _linear(x=None, wq=None, scale=None, **k):
    return st.st_int8_linear(dev(5, 16) if x is None else x, I8 if wq is None else wq, dev(7) if scale is None else scale, **k)


def _backward(**k):
    a = dict(x=dev(5, 16), w=dev(7, 16), dy=dev(5, 7), y=dev(5, 7), dx=dev(5, 16), dw=dev(7, 16), db=dev(7))
    a.update(k)
    return st.st_int8_linear_backward(**a)


def _quantize(**k):
    return st.st_int8_quantize(**dict(dict(x=dev(5, 16)), **k))


def _tensors(**k):
    a = dict(params=[dev(300), dev(2, 2)], grads=[dev(300), dev(4)], m=[dev(300, dtype=torch.int8), dev(4, dtype=torch.int8)],
             v=[dev(300, dtype=torch.uint8), dev(4, dtype=torch.uint8)], m_scales=[dev(2), dev(1)], v_scales=[dev(2), dev(1)],
             copies=[dev(300, dtype=torch.bfloat16), dev(4, dtype=torch.bfloat16)], weight_decay=[0.1, 0.0])
    a.update(k)
    return st.AdamWTensors(**a)


def _step(**k):
    return st.st_adamw_step(_tensors(), 1, 0.1, **dict(dict(max_norm=1.0), **k))


def _state(**k):
    a = dict(m=dev(300, dtype=torch.int8), m_scale=dev(2), v=dev(300, dtype=torch.uint8), v_scale=dev(2), m_out=dev(300), v_out=dev(300))
    a.update(k)
    return st.st_adamw_state(**a)


HALF, BYTES = torch.float16, torch.int8
SHAPE, ARG, SPACE = st.ST_ERR_SHAPE, st.ST_ERR_ARG, st.ST_ERR_WORKSPACE
WRONG = {
    "quantize": (_quantize, "st_int8_quantize", [
        (dict(x=dev(5, 16, dtype=HALF)), ARG), (dict(x=torch.zeros(5, 16)), ARG), (dict(q=dev(4, 16, dtype=BYTES)), SHAPE),
        (dict(q=dev(5, 15, dtype=BYTES)), SHAPE), (dict(q=dev(5, 16)), SHAPE), (dict(q=dev(16, 5, dtype=BYTES).t()), SHAPE),
        (dict(q=torch.zeros(5, 16, dtype=BYTES)), ARG), (dict(scale=dev(4)), SHAPE), (dict(scale=dev(5, dtype=torch.bfloat16)), SHAPE),
        (dict(scale=dev(5, 2)[:, 0]), SHAPE), (dict(scale=torch.zeros(5)), ARG),
        (dict(x=dev(16, 5).t(), workspace=dev(8)), SPACE), (dict(x=dev(16, 5).t(), workspace=torch.zeros(1 << 20)), SPACE)]),
    "linear": (_linear, "st_int8_linear", [
        (dict(x=dev(5, 16, dtype=HALF)), ARG), (dict(x=torch.zeros(5, 16)), ARG), (dict(x=dev(5, 17)), SHAPE),
        (dict(wq=dev(7, 15, dtype=BYTES)), SHAPE), (dict(wq=dev(16, 7, dtype=BYTES).t()), SHAPE), (dict(wq=torch.zeros(7, 16, dtype=BYTES)), ARG),
        (dict(wq=dev(8, 16, dtype=BYTES)), SHAPE), (dict(scale=dev(6)), SHAPE), (dict(scale=dev(7, dtype=torch.float64)), SHAPE),
        (dict(scale=torch.zeros(7)), ARG), (dict(bias=dev(8)), SHAPE), (dict(bias=dev(7, dtype=torch.bfloat16)), SHAPE), (dict(bias=torch.zeros(7)), ARG),
        (dict(out=dev(5, 8)), SHAPE), (dict(out=dev(4, 7)), SHAPE), (dict(out=dev(7, 5).t()), SHAPE), (dict(out=dev(5, 7, dtype=HALF)), ARG),
        (dict(out=torch.zeros(5, 7)), ARG), (dict(out_dtype=HALF), ARG), (dict(workspace=dev(8)), SPACE), (dict(workspace=torch.zeros(1 << 20)), SPACE)]),
    "backward": (_backward, "st_int8_linear_backward", [
        *[(dict([(k, t)]), s) for k, n, m in (("x", 5, 16), ("w", 7, 16), ("dy", 5, 7), ("y", 5, 7))
          for t, s in ((dev(n, m, dtype=HALF), ARG), (torch.zeros(n, m), ARG), (dev(n, m, 1), SHAPE))],
        (dict(dx=dev(5, 15)), SHAPE), (dict(dx=dev(4, 16)), SHAPE), (dict(dx=dev(16, 5).t()), SHAPE), (dict(dx=dev(5, 16, dtype=HALF)), ARG),
        (dict(dx=torch.zeros(5, 16)), ARG), (dict(dw=dev(7, 15)), SHAPE), (dict(dw=dev(8, 16)), SHAPE), (dict(dw=dev(16, 7).t()), SHAPE),
        (dict(dw=dev(7, 16, dtype=torch.bfloat16)), ARG), (dict(dw=torch.zeros(7, 16)), ARG), (dict(db=dev(8)), SHAPE),
        (dict(db=dev(7, dtype=torch.bfloat16)), SHAPE), (dict(db=torch.zeros(7)), ARG), (dict(workspace=dev(8)), SPACE),
        (dict(workspace=torch.zeros(1 << 20)), SPACE)]),
    "list": (lambda **k: st.st_adamw_step(_tensors(**k), 1, 0.1), "st_adamw_step", [
        (dict(grads=[dev(300)]), SHAPE), (dict(grads=[dev(300), dev(5)]), SHAPE), (dict(grads=[dev(300), dev(4, dtype=torch.bfloat16)]), SHAPE),
        (dict(params=[dev(300, dtype=HALF), dev(4, dtype=HALF)]), ARG), (dict(params=[dev(300), dev(2, 2, 2)[:, :, 0]]), SHAPE),
        (dict(m=[dev(300), dev(4)]), SHAPE), (dict(v=[dev(300, dtype=BYTES), dev(4, dtype=BYTES)]), SHAPE), (dict(m_scales=None), SHAPE),
        (dict(v_scales=[dev(1), dev(1)]), SHAPE), (dict(m_scales=[dev(2), dev(2)]), SHAPE), (dict(m_scales=[dev(2, dtype=torch.int32), dev(1)]), SHAPE),
        (dict(copies=[dev(300), dev(4)]), SHAPE), (dict(copies=[dev(300, dtype=torch.bfloat16)]), SHAPE), (dict(weight_decay=[0.1]), SHAPE),
        (dict(params=[torch.zeros(300), dev(4)]), ARG), (dict(v_scales=[dev(2), torch.zeros(1)]), ARG)]),
    "step": (_step, "st_adamw_step", [
        (dict(grad_norm=dev(2)), SHAPE), (dict(grad_norm=dev(1, dtype=torch.float64)), SHAPE), (dict(grad_norm=torch.zeros(1)), ARG),
        (dict(workspace=dev(8)), SPACE), (dict(workspace=torch.zeros(1 << 20)), SPACE)]),
    "state": (_state, "st_adamw_state", [
        (dict(m=dev(299, dtype=BYTES)), SHAPE), (dict(v=dev(301, dtype=torch.uint8)), SHAPE), (dict(m=dev(300, 2, dtype=BYTES)[:, 0]), SHAPE),
        (dict(m_scale=dev(1)), SHAPE), (dict(v_scale=dev(2, 2)[:, 0]), SHAPE), (dict(m=torch.zeros(300, dtype=BYTES)), ARG),
        (dict(v_scale=torch.zeros(2)), ARG), (dict(m_out=dev(300, dtype=torch.bfloat16)), SHAPE), (dict(v_out=dev(300, 2)[:, 0]), SHAPE),
        (dict(v_out=torch.zeros(300)), ARG)]),
}


@pytest.mark.parametrize("name,at", [(name, i) for name, (_, _, wrong) in WRONG.items() for i in range(-1, len(wrong))])
def test_one_wrong_argument_is_refused(name, at, library):
    """The call as it is reaches the library; with one argument wrong it does not, and the status says what kind of fault it is."""
    call, entry, wrong = WRONG[name]
    if at < 0:
        call()
        assert [n for n, _ in library.calls] == [entry]
    else:
        refused(wrong[at][1], lambda: call(**wrong[at][0]), library)


@pytest.mark.parametrize("name", WRONG)
def test_the_librarys_own_refusals_are_raised(name, library, monkeypatch):
    call, entry, _ = WRONG[name]
    monkeypatch.setattr(library, entry, lambda *a: st.ST_ERR_HIP, raising=False)
    refused(st.ST_ERR_HIP, call, library)


def test_sizes_that_have_no_workspace_are_refused(library):
    long = st.ST_INT8_MAX_SUM + 1
    refused(SHAPE, lambda: st.new_int8_workspace(1, 1, long), library)
    refused(SHAPE, lambda: st.new_int8_workspace(1, 0, 4, backward=True), library)
    refused(SHAPE, lambda: st.st_int8_linear(dev(2, long), dev(3, long, dtype=BYTES), dev(3)), library)
    refused(ARG, lambda: st.new_adamw_state([dev(4)], bits=16), library)
