"""What the binding of the dense layers and of the AdamW step checks and makes before it calls the library, without a GPU.

The tensors are host tensors that say they are on a device, and the entry points are stand-ins that record their arguments (other
functions, those that give sizes among them, are the library's own): a call that gets through reaches the stand-in and nothing else.
"""
import pytest

import paper_2003_10735_amd as st

torch = pytest.importorskip("torch")


class OnDevice(torch.Tensor):
    is_cuda = True


ENTRY_POINTS = ("st_int8_quantize", "st_int8_linear", "st_int8_linear_backward", "st_adamw_step", "st_adamw_state")


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
