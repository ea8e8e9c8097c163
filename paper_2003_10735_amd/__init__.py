"""Thin Python binding of libshadowtutor_head.so (hand-written HIP for MI355X / gfx950).

Argument marshalling only: torch tensors supply device memory and the stream; every step of
the partial-distillation path runs inside the library's kernels.  There is no CPU fallback:
if the shared library is missing, importing the entry points raises.

Function names mirror the C ABI declared in include/shadowtutor_head.h.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from functools import lru_cache

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libshadowtutor_head.so")

ST_OK = 0
ST_ERR_NULL, ST_ERR_SHAPE, ST_ERR_ARG, ST_ERR_WORKSPACE, ST_ERR_HIP, ST_ERR_NO_DEVICE, ST_ERR_TOO_LARGE = -1, -2, -3, -4, -5, -6, -7
ST_NOALLOC_MAX_WORKSPACE_MIB = 96
ST_OBJECT_WEIGHTS_MAX_RADIUS = 32
ST_F32, ST_BF16 = 0, 1
ST_NCHW, ST_NHWC = 0, 1
ST_COMPUTE_F32, ST_COMPUTE_BF16 = 0, 1
ST_OPTIM_SGD, ST_OPTIM_ADAM = 0, 1
ST_ACT_NONE, ST_ACT_RELU, ST_ACT_GELU, ST_ACT_GELU_TANH, ST_ACT_SILU = 0, 1, 2, 3, 4
ST_LINEAR_MAX_CHANNELS = 1048576
ST_INT8_MAX_SUM = 131071
ST_ADAMW_BLOCK = 256

EXPORTS = ["st_num_params", "st_workspace_bytes", "st_head_forward", "st_head_forward_noalloc", "st_partial_distill",
           "st_miou", "st_object_weights", "st_strerror", "st_last_hip_error", "st_version",
           "st_get_workspace_layout", "st_profile_enable", "st_profile_filter", "st_profile_reset", "st_profile_read",
           "st_next_stride", "st_schedule_bounds", "st_schedule_total_time",
           "st_graph_cache_clear", "st_graph_cache_size", "st_metric_polling",
           "st_int8_quantize_workspace", "st_int8_quantize", "st_int8_linear_workspace", "st_int8_linear",
           "st_int8_linear_backward_workspace", "st_int8_linear_backward", "st_adamw_workspace", "st_adamw_step", "st_adamw_state",
           "st_linear_workspace", "st_linear", "st_linear_backward_workspace", "st_linear_backward", "st_grad_clip_workspace", "st_grad_clip"]


class StHeadDesc(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("n", "c_in", "h", "w", "c1", "c2", "n_classes", "upscale",
                                          "feat_dtype", "feat_layout", "compute", "ignore_index",
                                          "grouped")]


class StDistillOpts(C.Structure):
    _fields_ = [("momentum", C.c_float), ("velocity", C.c_void_p), ("threshold", C.c_double),
                ("strict_break", C.c_int32), ("return_best", C.c_int32),
                ("optimizer", C.c_int32), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("adam_m", C.c_void_p), ("adam_v", C.c_void_p), ("adam_t0", C.c_int32),
                ("pixel_weights", C.c_void_p), ("feature_grad", C.c_void_p), ("use_graph", C.c_int32),
                ("best_params", C.c_void_p), ("expect_key_frame", C.c_int32)]


class StScheduleParams(C.Structure):
    _fields_ = [(k, C.c_double) for k in ("t_si", "t_sd", "t_ti", "t_net", "s_net", "min_stride",
                                          "max_stride", "max_updates")]


class StScheduleBounds(C.Structure):
    _fields_ = [(k, C.c_double) for k in ("t_c_lower", "t_c_upper", "traffic_lower", "traffic_upper",
                                          "throughput_lower", "throughput_upper")]


class StDistillResult(C.Structure):
    _fields_ = [("losses", C.c_void_p), ("mious", C.c_void_p), ("confusion", C.c_void_p),
                ("pred", C.c_void_p), ("steps_taken", C.c_int32), ("best_metric", C.c_double),
                ("first_metric", C.c_double)]


class StWorkspaceLayout(C.Structure):
    _fields_ = [(k, C.c_size_t) for k in ("feat", "a1", "a2", "da1", "da2", "z", "g", "theta",
                                           "grad", "elem_size", "total", "row_pitch", "grad_copies",
                                           "grad_stride")] + [("splits", C.c_size_t * 3)]


class StMatrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64),
                ("row_stride", C.c_int64), ("col_stride", C.c_int64)]


class StAdamwTensor(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [
        ("n", C.c_int64), ("weight_decay", C.c_double)]


class StAdamwOpts(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("param_dtype", "grad_dtype", "state_bits", "t")] + [
        (k, C.c_double) for k in ("lr", "beta1", "beta2", "eps", "grad_scale", "max_norm")] + [("grad_norm", C.c_void_p)]


class StLinearOpts(C.Structure):
    _fields_ = [("bias", C.c_void_p), ("activation", C.c_int32), ("residual_dtype", C.c_int32), ("residual", C.c_void_p),
                ("residual_pitch", C.c_int64), ("pre", C.c_void_p), ("pre_pitch", C.c_int64), ("pre_dtype", C.c_int32)]


class StLinearGrads(C.Structure):
    _fields_ = [("dx", C.c_void_p), ("dx_pitch", C.c_int64), ("dx_dtype", C.c_int32), ("dw_dtype", C.c_int32), ("dw", C.c_void_p),
                ("dw_pitch", C.c_int64), ("db", C.c_void_p), ("accumulate", C.c_int32)]


class StGradTensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("grad_dtype", C.c_int32), ("out_dtype", C.c_int32)]


class StKernelStat(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int64), ("total_ms", C.c_double)]


class DistillReturn(tuple):
    """(steps_taken, best_metric or None) of st_partial_distill; with a threshold also
    `.first_metric`, the metric before any update."""
    first_metric = None


class StError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().st_strerror(status).decode()
        extra = f" (hipError {lib().st_last_hip_error()})" if status == ST_ERR_HIP else ""
        super().__init__(f"{where}: {msg}{extra} [status {status}]")


_LIB = None


def lib():
    """The loaded shared library.  Raises if it has not been built (no fallback exists)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2003_10735_amd.build` "
                "(hipcc, gfx950).  There is no CPU fallback.")
        L = C.CDLL(LIB_PATH)
        L.st_num_params.restype = C.c_size_t
        L.st_num_params.argtypes = [C.POINTER(StHeadDesc)]
        L.st_workspace_bytes.restype = C.c_size_t
        L.st_workspace_bytes.argtypes = [C.POINTER(StHeadDesc)]
        L.st_head_forward.restype = C.c_int
        L.st_head_forward.argtypes = [C.POINTER(StHeadDesc), C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_void_p]
        L.st_head_forward_noalloc.restype = C.c_int
        L.st_head_forward_noalloc.argtypes = [C.POINTER(StHeadDesc), C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p]
        L.st_partial_distill.restype = C.c_int
        L.st_partial_distill.argtypes = [C.POINTER(StHeadDesc), C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_int32, C.c_float, C.POINTER(StDistillOpts),
                                         C.POINTER(StDistillResult), C.c_void_p, C.c_void_p]
        L.st_miou.restype = C.c_int
        L.st_miou.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p,
                              C.c_void_p, C.c_void_p]
        L.st_object_weights.restype = C.c_int
        L.st_object_weights.argtypes = [C.c_void_p] + [C.c_int32] * 8 + [C.c_void_p, C.c_void_p]
        L.st_strerror.restype = C.c_char_p
        L.st_strerror.argtypes = [C.c_int]
        L.st_last_hip_error.restype = C.c_int
        L.st_version.restype = C.c_char_p
        L.st_get_workspace_layout.restype = C.c_int
        L.st_get_workspace_layout.argtypes = [C.POINTER(StHeadDesc), C.POINTER(StWorkspaceLayout)]
        L.st_next_stride.restype = C.c_double
        L.st_next_stride.argtypes = [C.c_double] * 5
        L.st_schedule_bounds.restype = C.c_int
        L.st_schedule_bounds.argtypes = [C.POINTER(StScheduleParams), C.POINTER(StScheduleBounds)]
        L.st_schedule_total_time.restype = C.c_double
        L.st_schedule_total_time.argtypes = [C.POINTER(StScheduleParams)] + [C.c_double] * 4
        i32, i64, ptr, size = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t
        for name, result, args in (
                ("st_int8_quantize_workspace", size, [i64, i64]),
                ("st_int8_quantize", C.c_int, [ptr, ptr, i64, ptr, ptr, ptr]),
                ("st_int8_linear_workspace", size, [i64, i64, i64]),
                ("st_int8_linear", C.c_int, [ptr, ptr, i64, ptr, i64, ptr, i32, ptr, i32, i64, ptr, ptr]),
                ("st_int8_linear_backward_workspace", size, [i64, i64, i64]),
                ("st_int8_linear_backward", C.c_int, [ptr, ptr, ptr, ptr, ptr, i32, i64, ptr, i64, ptr, ptr, ptr]),
                ("st_adamw_workspace", size, [ptr, i32]),
                ("st_adamw_step", C.c_int, [ptr, i32, ptr, ptr, ptr]),
                ("st_adamw_state", C.c_int, [ptr, ptr, ptr, ptr, i64, ptr, ptr, ptr]),
                ("st_linear_workspace", size, [ptr, ptr]),
                ("st_linear", C.c_int, [ptr, ptr, ptr, ptr, i32, i64, ptr, size, ptr]),
                ("st_linear_backward_workspace", size, [ptr, ptr, ptr, i32]),
                ("st_linear_backward", C.c_int, [ptr, ptr, ptr, ptr, i32, ptr, ptr, size, ptr]),
                ("st_grad_clip_workspace", size, [ptr, i32]),
                ("st_grad_clip", C.c_int, [ptr, i32, C.c_double, C.c_double, ptr, ptr, ptr])):
            f = getattr(L, name)
            f.restype, f.argtypes = result, args
        L.st_graph_cache_size.restype = C.c_int
        L.st_profile_enable.argtypes = [C.c_int]
        L.st_profile_filter.argtypes = [C.c_char_p]
        L.st_profile_read.restype = C.c_int
        L.st_profile_read.argtypes = [C.POINTER(StKernelStat), C.c_int]
        _LIB = L
    return _LIB


@dataclass
class HeadDesc:
    n: int
    c_in: int
    h: int
    w: int
    c1: int
    c2: int
    n_classes: int
    feat_dtype: int = ST_BF16
    compute: int = ST_COMPUTE_BF16
    ignore_index: int = -1
    upscale: int = 8
    feat_layout: int = ST_NCHW
    grouped: int = 0        # 1: n heads, one per frame; per-head arrays are [n, ...]

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        self.__dict__.pop("_struct", None)

    def _ref(self):
        """A reference to this descriptor's C struct for the calls below, which only read it (built once,
        again after a field has changed: filling thirteen fields costs more than the call)."""
        struct = self.__dict__.get("_struct")
        if struct is None:
            struct = self.__dict__["_struct"] = self.c()
        return C.byref(struct)

    def c(self) -> StHeadDesc:
        return StHeadDesc(self.n, self.c_in, self.h, self.w, self.c1, self.c2, self.n_classes,
                          self.upscale, self.feat_dtype, self.feat_layout, self.compute,
                          self.ignore_index, self.grouped)

    @staticmethod
    def of(wl) -> "HeadDesc":
        """Descriptor of a workloads.Workload."""
        return HeadDesc(wl.n, wl.c_in, wl.h, wl.w, wl.c1, wl.c2, wl.n_classes,
                        ST_BF16 if wl.feat_dtype == "bf16" else ST_F32,
                        ST_COMPUTE_BF16 if wl.compute == "bf16" else ST_COMPUTE_F32,
                        wl.ignore_index)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _addr(t):
    """Device address of a tensor as the integer that ctypes takes for a pointer argument or field."""
    return None if t is None else t.data_ptr()


_RAW_STREAM = None


def _stream(stream):
    """The stream's handle as an integer (the current stream of the current device if none is given).  The handle is asked for without
    the object around it, which takes longer to make than a launch."""
    global _RAW_STREAM
    if stream is not None:
        return stream.cuda_stream
    if _RAW_STREAM is None:
        import torch
        torch.cuda.current_stream()         # initialises the device
        _RAW_STREAM = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    return _RAW_STREAM[0](_RAW_STREAM[1]())


def _own(stream, make, result=False):
    """A tensor that a call makes itself.  Where the call is given a stream, the tensor is made on that stream: the allocator then neither
    takes memory that another stream's work still uses nor hands this on while the call's work is under way.  A result may be used on
    the caller's current stream as well."""
    if stream is None:
        return make()
    import torch
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)):
        t = make()
    if result:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _check(status: int, where: str):
    if status != ST_OK:
        raise StError(status, where)


def st_num_params(desc: HeadDesc) -> int:
    d = desc.c()
    return int(lib().st_num_params(C.byref(d)))


def st_workspace_bytes(desc: HeadDesc) -> int:
    d = desc.c()
    return int(lib().st_workspace_bytes(C.byref(d)))


def st_get_workspace_layout(desc: HeadDesc) -> dict:
    d, out = desc.c(), StWorkspaceLayout()
    _check(lib().st_get_workspace_layout(C.byref(d), C.byref(out)), "st_get_workspace_layout")
    return {k: ([int(v) for v in getattr(out, k)] if k == "splits" else int(getattr(out, k)))
            for k, _ in StWorkspaceLayout._fields_}


def new_workspace(desc: HeadDesc, device="cuda"):
    """A device buffer of st_workspace_bytes(desc) bytes (torch allocations are 256-byte aligned)."""
    import torch
    nbytes = st_workspace_bytes(desc)
    if nbytes == 0:
        raise StError(ST_ERR_SHAPE, "st_workspace_bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def st_head_forward(desc: HeadDesc, features, head_params, logits_lowres=None, pred=None,
                    workspace=None, stream=None):
    """features [n,c_in,h,w] (float32 or bfloat16 cuda tensor), head_params float32 [num_params]
    ([n, num_params] for a grouped descriptor).  Fills logits_lowres [n,C,h,w] float32 and/or pred [n,8h,8w] uint8 when given."""
    ws = workspace if workspace is not None else _own(stream, lambda: new_workspace(desc, features.device))
    _check(lib().st_head_forward(desc._ref(), _addr(features), _addr(head_params), _addr(logits_lowres), _addr(pred),
                                 _addr(ws), _stream(stream)), "st_head_forward")
    return logits_lowres, pred


def st_head_forward_noalloc(desc: HeadDesc, features, head_params, logits_lowres=None, pred=None, stream=None):
    """st_head_forward on the library's built-in scratch: no workspace argument, no allocation."""
    _check(lib().st_head_forward_noalloc(desc._ref(), _addr(features), _addr(head_params), _addr(logits_lowres),
                                         _addr(pred), _stream(stream)), "st_head_forward_noalloc")
    return logits_lowres, pred


def st_partial_distill(desc: HeadDesc, features, teacher_labels, head_params, steps: int, lr: float,
                       momentum: float = 0.0, velocity=None, threshold: float = 0.0,
                       strict_break: bool = True, return_best: bool = False, losses=None,
                       mious=None, confusion=None, pred=None, workspace=None, stream=None,
                       adam=None, pixel_weights=None, feature_grad=None, graph=False, best_params=None,
                       expect_key_frame=False):
    """Runs the library's st_partial_distill; head_params (and the optimiser state) are updated
    in place.  `adam` = dict(m=, v=, t0=0, beta1=0.9, beta2=0.999, eps=1e-8) selects Adam;
    `pixel_weights` (uint8 [n,8h,8w]) scales every pixel's loss; `feature_grad` (float32
    [n,c_in,h,w]) receives d loss / d features of the last backward pass; `best_params` (float32,
    like head_params) receives Algorithm 1's best parameters when a threshold is given.
    With a grouped descriptor head_params and the optimiser state are [n, num_params] and losses
    [steps+1, n].  graph=True launches the call through the library's cached HIP graph
    (st_distill_opts.use_graph).  expect_key_frame=True (with a threshold) makes the first pass compute its
    gradients at once instead of scoring first (st_distill_opts.expect_key_frame).
    Returns (steps_taken, best_metric or None); with a threshold the returned tuple also carries
    `.first_metric`, the metric before any update."""
    ws = workspace if workspace is not None else _own(stream, lambda: new_workspace(desc, features.device))
    opts = None
    if (momentum != 0.0 or threshold > 0.0 or velocity is not None or adam is not None or pixel_weights is not None
            or feature_grad is not None or graph or best_params is not None or expect_key_frame):
        # (fields start as zeros: only what differs is filled in)
        o = StDistillOpts()
        o.momentum, o.threshold, o.strict_break = momentum, threshold, 1 if strict_break else 0
        if return_best:
            o.return_best = 1
        if velocity is not None:
            o.velocity = velocity.data_ptr()
        if pixel_weights is not None:
            o.pixel_weights = pixel_weights.data_ptr()
        if feature_grad is not None:
            o.feature_grad = feature_grad.data_ptr()
        if graph:
            o.use_graph = 1
        if best_params is not None:
            o.best_params = best_params.data_ptr()
        if expect_key_frame:
            o.expect_key_frame = 1
        if adam is not None:
            o.optimizer = ST_OPTIM_ADAM
            o.beta1, o.beta2 = adam.get("beta1", 0.9), adam.get("beta2", 0.999)
            o.eps = adam.get("eps", 1e-8)
            o.adam_m, o.adam_v = _addr(adam["m"]), _addr(adam["v"])
            o.adam_t0 = int(adam.get("t0", 0))
        opts = C.byref(o)
    res = StDistillResult(_addr(losses), _addr(mious), _addr(confusion), _addr(pred))
    _check(lib().st_partial_distill(desc._ref(), _addr(features), _addr(teacher_labels), _addr(head_params), steps, lr,
                                    opts, C.byref(res), _addr(ws), _stream(stream)), "st_partial_distill")
    ret = DistillReturn((res.steps_taken, res.best_metric if threshold > 0.0 else None))
    ret.first_metric = res.first_metric if threshold > 0.0 else None
    return ret


def st_miou(pred, labels, n_classes: int, ignore_index: int = -1, confusion=None, miou=None,
            stream=None):
    """pred uint8 [..], labels int32 [..] cuda tensors.  Returns (confusion int64 [C,C], miou float64 [1])."""
    if confusion is None or miou is None:
        import torch
        if confusion is None:
            confusion = _own(stream, lambda: torch.empty((n_classes, n_classes), dtype=torch.int64, device=pred.device), result=True)
        if miou is None:
            miou = _own(stream, lambda: torch.empty(1, dtype=torch.float64, device=pred.device), result=True)
    _check(lib().st_miou(_addr(pred), _addr(labels), pred.numel(), n_classes, ignore_index,
                         confusion.data_ptr(), miou.data_ptr(), _stream(stream)), "st_miou")
    return confusion, miou


def st_object_weights(labels, n_classes: int, radius: int, factor: int = 5, background: int = 0,
                      ignore_index: int = -1, weights=None, stream=None):
    """labels int32 [n, H, W] cuda tensor -> uint8 [n, H, W] loss weights (`factor` within `radius`
    pixels of an object label, 1 elsewhere): the `pixel_weights` of st_partial_distill."""
    n, H, W = labels.shape
    if weights is None:
        import torch
        weights = _own(stream, lambda: torch.empty((n, H, W), dtype=torch.uint8, device=labels.device), result=True)
    _check(lib().st_object_weights(labels.data_ptr(), n, H, W, n_classes, background, ignore_index, radius, factor,
                                   weights.data_ptr(), _stream(stream)), "st_object_weights")
    return weights


# ---------------------------------------------------------------- dense layers in 8-bit integers
_DTYPES = _INT8 = None


def _types():
    global _DTYPES, _INT8
    import torch
    _INT8 = torch.int8
    _DTYPES = {torch.float32: ST_F32, torch.bfloat16: ST_BF16}
    return _DTYPES


def _dtype(t, where):
    """ST_F32 or ST_BF16 of a tensor."""
    d = (_DTYPES or _types()).get(t.dtype)
    if d is None:
        raise StError(ST_ERR_ARG, where)
    return d


def _matrix(t, where):
    """A two-dimensional tensor as the library takes it: either of its strides 1."""
    if t is None:
        raise StError(ST_ERR_NULL, where)
    shape = t.shape
    if len(shape) != 2:
        raise StError(ST_ERR_SHAPE, where)
    if not t.is_cuda:
        raise StError(ST_ERR_ARG, where)
    return StMatrix(t.data_ptr(), _dtype(t, where), *shape, *t.stride())


def _out_matrix(t, rows, cols, where):
    """Checks a result that lies row by row; returns its pitch."""
    if t.shape != (rows, cols):
        raise StError(ST_ERR_SHAPE, where)
    if not t.is_cuda:
        raise StError(ST_ERR_ARG, where)
    pitch, step = t.stride()
    if step != 1 and cols > 1:
        raise StError(ST_ERR_SHAPE, where)
    return pitch if rows > 1 or pitch > cols else cols


def _float_vector(t, n, where):
    if t is None:
        raise StError(ST_ERR_NULL, where)
    if t.numel() != n or not t.is_contiguous() or (_DTYPES or _types()).get(t.dtype) != ST_F32:
        raise StError(ST_ERR_SHAPE, where)
    if not t.is_cuda:
        raise StError(ST_ERR_ARG, where)
    return t.data_ptr()


def _scratch(nbytes, device, where):
    import torch
    if nbytes == 0:
        raise StError(ST_ERR_SHAPE, where)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


@lru_cache(maxsize=1024)
def _int8_bytes(m: int, n: int, k: int, backward: bool) -> int:
    """Bytes of scratch that the sizes ask for; 0: they are refused."""
    return (lib().st_int8_linear_backward_workspace if backward else lib().st_int8_linear_workspace)(m, n, k)


def _given(ws, nbytes, where):
    """Address of a caller's scratch of at least `nbytes` (where sizes are refused, 0, the library says so)."""
    if not ws.is_cuda or ws.nbytes < nbytes:
        raise StError(ST_ERR_WORKSPACE, where)
    return ws.data_ptr()


def int8_pitch(cols: int) -> int:
    """Bytes of a row of `cols` 8-bit integers: a multiple of 16."""
    return (cols + 15) // 16 * 16


def new_int8_workspace(m: int, n: int, k: int, backward: bool = False, device="cuda"):
    """Scratch for st_int8_linear (or with backward=True st_int8_linear_backward) of m tokens, k -> n channels."""
    return _scratch(_int8_bytes(m, n, k, bool(backward)), device, "new_int8_workspace")


def st_int8_quantize(x, q=None, scale=None, workspace=None, stream=None):
    """Rows of x [rows, cols] (float32 or bfloat16, row by row or column by column; x.t() quantises the columns) as 8-bit integers:
    (q int8 [rows, int8_pitch(cols)], scale float32 [rows]).  A row's bytes from cols up to the next multiple of 128 become zeros as far
    as the step between two rows of q reaches; a q that is too narrow to hold them (a part of a wider matrix's columns) is refused."""
    import torch
    where = "st_int8_quantize"
    mx = _matrix(x, where)
    rows, cols = x.shape
    if q is None:
        q = _own(stream, lambda: torch.empty((rows, int8_pitch(cols)), dtype=torch.int8, device=x.device), result=True)
    if scale is None:
        scale = _own(stream, lambda: torch.empty(rows, dtype=torch.float32, device=x.device), result=True)
    if q.dim() != 2 or q.shape[0] != rows or q.dtype != torch.int8 or q.stride(1) != 1:
        raise StError(ST_ERR_SHAPE, where)
    pitch = q.stride(0) if rows > 1 else q.shape[1]
    if q.shape[1] < max(cols, min((cols + 127) // 128 * 128, pitch)):
        raise StError(ST_ERR_SHAPE, where)
    if not q.is_cuda:
        raise StError(ST_ERR_ARG, where)
    ws = workspace
    if cols > 1 and mx.col_stride != 1:
        nbytes = lib().st_int8_quantize_workspace(rows, cols)
        if ws is None:
            ws = _own(stream, lambda: _scratch(nbytes, x.device, where))
        _given(ws, nbytes, where)
    _check(lib().st_int8_quantize(C.byref(mx), q.data_ptr(), pitch, _float_vector(scale, rows, where),
                                  _addr(ws), _stream(stream)), where)
    return q, scale


def st_int8_linear(x, wq, w_scale, bias=None, relu: bool = False, out=None, out_dtype=None, workspace=None, stream=None):
    """out [m, n] = act(x W^T + bias): x [m, k] float32 or bfloat16, row by row or column by column, its rows (tokens) quantised within
    the call; W as st_int8_quantize(W) leaves it: wq int8 [n, >= k], w_scale float32 [n].  out: float32 or bfloat16, as given, else of
    out_dtype, else of x's type."""
    where = "st_int8_linear"
    mx = _matrix(x, where)
    m, k = mx.rows, mx.cols
    if wq is None:
        raise StError(ST_ERR_NULL, where)
    if wq.dim() != 2:
        raise StError(ST_ERR_SHAPE, where)
    n, width = wq.shape
    w_pitch, step = wq.stride()
    if width < k or step != 1 or wq.dtype != _INT8:
        raise StError(ST_ERR_SHAPE, where)
    if not wq.is_cuda:
        raise StError(ST_ERR_ARG, where)
    if out is None:
        import torch
        out = _own(stream, lambda: torch.empty((m, n), dtype=out_dtype or x.dtype, device=x.device), result=True)
    pitch = _out_matrix(out, m, n, where)
    if workspace is None:
        workspace = _own(stream, lambda: new_int8_workspace(m, n, k, device=x.device))
    status = (_LIB or lib()).st_int8_linear(
        C.byref(mx), wq.data_ptr(), w_pitch if n > 1 else width, _float_vector(w_scale, n, where), n,
        None if bias is None else _float_vector(bias, n, where), 1 if relu else 0, out.data_ptr(), _dtype(out, where), pitch,
        _given(workspace, _int8_bytes(m, n, k, False), where), _stream(stream))
    if status:
        raise StError(status, where)
    return out


def st_int8_linear_backward(x, w, dy, y=None, dx=None, dw=None, db=None, workspace=None, stream=None):
    """Gradients of a dense layer, both products in 8-bit integers: dx [m, k] (float32 or bfloat16) = dz W, dw [n, k] float32 = dz^T x,
    db [n] float32 = sum of dz, where dz = dy, or with y (the layer's result, a layer with ReLU) dy where y > 0.  Only the outputs that
    are given are computed; x may be None without dw, w without dx.  x, w (float weights), dy, y: float32 or bfloat16, row by row or column by
    column, y as dy (one token: with any step).  Returns (dx, dw, db)."""
    where = "st_int8_linear_backward"
    mdy = _matrix(dy, where)
    m, n = mdy.rows, mdy.cols
    mx, mw, my = (None if t is None else _matrix(t, where) for t in (x, w, y))
    if (dx is not None and w is None) or (dw is not None and x is None):
        raise StError(ST_ERR_NULL, where)
    k = mw.cols if dx is not None else mx.cols if dw is not None else 1
    dx_pitch = k if dx is None else _out_matrix(dx, m, k, where)
    if dw is not None and _dtype(dw, where) != ST_F32:
        raise StError(ST_ERR_ARG, where)
    dw_pitch = k if dw is None else _out_matrix(dw, n, k, where)
    ws = workspace if workspace is not None else _own(stream, lambda: new_int8_workspace(m, n, k, backward=True, device=dy.device))
    _check(lib().st_int8_linear_backward(*[None if a is None else C.byref(a) for a in (mx, mw, mdy, my)], _addr(dx),
                                         ST_F32 if dx is None else _dtype(dx, where), dx_pitch, _addr(dw), dw_pitch,
                                         None if db is None else _float_vector(db, n, where),
                                         _given(ws, _int8_bytes(m, n, k, True), where), _stream(stream)), where)
    return dx, dw, db


# ---------------------------------------------------------------- AdamW over many tensors
class AdamWTensors:
    """The list that st_adamw_step works on: parameters, gradients and states of the same lengths, contiguous, in a HOST array that is
    filled once (the tensors are kept alive with it).  params, grads: float32 or bfloat16, one type each; m, v: float32, or int8 and uint8
    codes with m_scales and v_scales (float32, one value for each ST_ADAMW_BLOCK values; new_adamw_state makes them); copies: bfloat16 or
    None; weight_decay: a number or one for each tensor."""

    def __init__(self, params, grads, m, v, m_scales=None, v_scales=None, copies=None, weight_decay=0.0):
        import torch
        where = "AdamWTensors"
        count = len(params)
        if any(t is None for x in (params, grads, m, v, m_scales, v_scales, copies) if x is not None for t in x):
            raise StError(ST_ERR_NULL, where)
        eight = count > 0 and m[0].dtype == torch.int8
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * count
        lists = [params, grads, m, v, m_scales, v_scales, copies]
        wanted = [params[0].dtype if count else None, grads[0].dtype if count else None, torch.int8 if eight else torch.float32,
                  torch.uint8 if eight else torch.float32, torch.float32, torch.float32, torch.bfloat16]
        if any(x is not None and len(x) != count for x in lists) or len(decay) != count or eight != (m_scales is not None) \
                or eight != (v_scales is not None):
            raise StError(ST_ERR_SHAPE, where)
        self.array = (StAdamwTensor * max(count, 1))()
        self.count, self.kept = count, [None if x is None else list(x) for x in lists]
        self.state_bits = 8 if eight else 32
        self.param_dtype, self.grad_dtype = (_dtype(params[0], where), _dtype(grads[0], where)) if count else (ST_F32, ST_F32)
        fields = [(name, x, dtype, name.endswith("scale")) for (name, _), x, dtype in zip(StAdamwTensor._fields_, lists, wanted)
                  if x is not None]
        for i, a in enumerate(self.array[:count]):
            n = params[i].numel()
            runs = (n + ST_ADAMW_BLOCK - 1) // ST_ADAMW_BLOCK
            for name, x, dtype, scale in fields:
                t = x[i]
                if t.dtype != dtype or t.numel() != (runs if scale else n) or not t.is_contiguous():
                    raise StError(ST_ERR_SHAPE, where)
                setattr(a, name, t.data_ptr())
            a.n, a.weight_decay = n, float(decay[i])
        self.device = params[0].device if count else "cuda"
        self._norm_bytes = None
        self.on_device = all(t.is_cuda for x in lists if x is not None for t in x)

    def norm_bytes(self) -> int:
        """Bytes of scratch that the norm of this list asks for."""
        if self._norm_bytes is None:
            self._norm_bytes = lib().st_adamw_workspace(self.array, self.count)
        return self._norm_bytes

    def set_grads(self, grads):
        """Other gradient tensors (of the same type and lengths) from the next step on."""
        grads, where = list(grads), "AdamWTensors"
        if len(grads) != self.count:
            raise StError(ST_ERR_SHAPE, where)
        for g, old in zip(grads, self.kept[1]):      # all of them before any is taken: a refused list changes nothing
            if g is None:
                raise StError(ST_ERR_NULL, where)
            if self.on_device and not g.is_cuda:
                raise StError(ST_ERR_ARG, where)
            if g.dtype != old.dtype or g.numel() != old.numel() or not g.is_contiguous():
                raise StError(ST_ERR_SHAPE, where)
        for a, g in zip(self.array, grads):
            a.grad = g.data_ptr()
        self.kept[1] = grads


def new_adamw_state(params, bits: int = 32):
    """Zeroed states for a list of tensors: dict(m=, v=) with bits = 32, dict(m=, v=, m_scales=, v_scales=) with bits = 8."""
    import torch
    if bits not in (8, 32):
        raise StError(ST_ERR_ARG, "new_adamw_state")
    if bits == 32:
        return {name: [torch.zeros(p.numel(), dtype=torch.float32, device=p.device) for p in params] for name in ("m", "v")}
    runs = [(p.numel() + ST_ADAMW_BLOCK - 1) // ST_ADAMW_BLOCK for p in params]
    state = {name: [torch.zeros(p.numel(), dtype=t, device=p.device) for p in params] for name, t in (("m", torch.int8), ("v", torch.uint8))}
    for name in ("m_scales", "v_scales"):
        state[name] = [torch.zeros(r, dtype=torch.float32, device=p.device) for r, p in zip(runs, params)]
    return state


def new_adamw_workspace(tensors: AdamWTensors):
    """Scratch for st_adamw_step's norm of this list."""
    return _scratch(tensors.norm_bytes(), tensors.device, "new_adamw_workspace")


def st_adamw_step(tensors: AdamWTensors, t: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                  max_norm: float = 0.0, grad_scale: float = 1.0, grad_norm=None, workspace=None, stream=None):
    """Step number t (from 1 on) of AdamW on every tensor of the list, in place.  max_norm > 0 clips by the norm of all (scaled)
    gradients, which grad_norm (float32 [1]) receives if given; a norm that is not finite then leaves everything as it was."""
    where = "st_adamw_step"
    if not tensors.on_device:
        raise StError(ST_ERR_ARG, where)
    ws = workspace
    if max_norm > 0.0 or grad_norm is not None:
        if ws is None:
            ws = _own(stream, lambda: new_adamw_workspace(tensors))
        _given(ws, tensors.norm_bytes(), where)
    o = StAdamwOpts(tensors.param_dtype, tensors.grad_dtype, tensors.state_bits, t, lr, beta1, beta2, eps, grad_scale, max_norm,
                    None if grad_norm is None else _float_vector(grad_norm, 1, where))
    _check(lib().st_adamw_step(tensors.array, tensors.count, C.byref(o), _addr(ws), _stream(stream)), where)


def st_adamw_state(m, m_scale, v, v_scale, m_out=None, v_out=None, stream=None):
    """The float32 values that a state in 8 bits (m int8, v uint8, scales float32) stands for, into m_out and v_out (made if neither is
    given).  Returns (m_out, v_out)."""
    import torch
    where = "st_adamw_state"
    if m_out is None and v_out is None:
        if m is None or v is None:
            raise StError(ST_ERR_NULL, where)
        m_out, v_out = (_own(stream, lambda: torch.empty(m.shape, dtype=torch.float32, device=m.device), result=True) for _ in range(2))
    n = (m_out if m_out is not None else v_out).numel()
    for codes, scale, out, dtype in ((m, m_scale, m_out, torch.int8), (v, v_scale, v_out, torch.uint8)):
        if out is not None and (codes is None or scale is None):
            raise StError(ST_ERR_NULL, where)
        if out is not None and (codes.numel() != n or codes.dtype != dtype or not codes.is_contiguous()
                                or scale.numel() * ST_ADAMW_BLOCK < n or not scale.is_contiguous() or scale.dtype != torch.float32):
            raise StError(ST_ERR_SHAPE, where)
        if out is not None and not (codes.is_cuda and scale.is_cuda):
            raise StError(ST_ERR_ARG, where)
    _check(lib().st_adamw_state(_addr(m) if m_out is not None else None, _addr(m_scale) if m_out is not None else None,
                                _addr(v) if v_out is not None else None, _addr(v_scale) if v_out is not None else None, n,
                                None if m_out is None else _float_vector(m_out, n, where),
                                None if v_out is None else _float_vector(v_out, n, where), _stream(stream)), where)
    return m_out, v_out


# ---------------------------------------------------------------- dense layers in bfloat16 or float32
# (a call's structs as bytes in one go: filling ctypes fields one by one costs a third of a microsecond each more)
_MATRIX_BYTES, _OPTS_BYTES, _GRADS_BYTES = struct.Struct("@Piqqqq"), struct.Struct("@PiiPqPqi4x"), struct.Struct("@PqiiPqPi4x")


def _packed(t, where):
    """A two-dimensional tensor as the bytes of an st_matrix, its rows and its columns."""
    if t is None:
        raise StError(ST_ERR_NULL, where)
    shape = t.shape
    if len(shape) != 2:
        raise StError(ST_ERR_SHAPE, where)
    if not t.is_cuda:
        raise StError(ST_ERR_ARG, where)
    rows, cols = shape
    return _MATRIX_BYTES.pack(t.data_ptr(), _dtype(t, where), rows, cols, *t.stride()), rows, cols


def new_linear_workspace(x, w, dy=None, activation: int = ST_ACT_NONE):
    """Scratch for st_linear on matrices that lie as x and w do, or with dy for st_linear_backward (x or w may then be None where the
    gradient that needs it is not asked for).  Most of it is for copies of matrices at odd addresses or with odd strides, and for dz."""
    where = "new_linear_workspace"
    like = x if x is not None else w if w is not None else dy
    if like is None or (dy is None and (x is None or w is None)):
        raise StError(ST_ERR_NULL, where)
    mx, mw, mdy = (None if t is None else _packed(t, where)[0] for t in (x, w, dy))
    nbytes = lib().st_linear_workspace(mx, mw) if dy is None else lib().st_linear_backward_workspace(mx, mw, mdy, activation)
    return _scratch(nbytes, like.device, where)


def _workspace(workspace, where):
    if not workspace.is_cuda:
        raise StError(ST_ERR_WORKSPACE, where)
    return workspace.data_ptr(), workspace.nbytes


def st_linear(x, w, bias=None, activation: int = ST_ACT_NONE, residual=None, pre=None, out=None, out_dtype=None, workspace=None, stream=None):
    """out [m, n] = act(x W^T + bias) + residual: x [m, k] and w [n, k] float32 or bfloat16, both of one type, row by row or column by
    column each at any distance (one stride is 1);
    bias float32 [n]; residual [m, n] float32 or bfloat16, row by row, which may be out itself.  pre [m, n] (float32 or bfloat16, row by
    row) receives x W^T + bias, which st_linear_backward asks for.  out: float32 or bfloat16, as given, else of out_dtype, else of x's type."""
    where = "st_linear"
    mx, m, _ = _packed(x, where)
    mw, n, _ = _packed(w, where)
    if out is None:
        import torch
        out = _own(stream, lambda: torch.empty((m, n), dtype=out_dtype or x.dtype, device=x.device), result=True)
    pitch = _out_matrix(out, m, n, where)
    opts = None
    if bias is not None or activation or residual is not None or pre is not None:
        r = (0, 0, 0) if residual is None else (residual.data_ptr(), _out_matrix(residual, m, n, where), _dtype(residual, where))
        z = (0, 0, 0) if pre is None else (pre.data_ptr(), _out_matrix(pre, m, n, where), _dtype(pre, where))
        opts = _OPTS_BYTES.pack(0 if bias is None else _float_vector(bias, n, where), activation, r[2], r[0], r[1], z[0], z[1], z[2])
    if workspace is None:
        workspace = _own(stream, lambda: new_linear_workspace(x, w))
    address, nbytes = _workspace(workspace, where)
    status = (_LIB or lib()).st_linear(mx, mw, opts, out.data_ptr(), _dtype(out, where), pitch, address, nbytes, _stream(stream))
    if status:
        raise StError(status, where)
    return out


def st_linear_backward(x, w, dy, pre=None, activation: int = ST_ACT_NONE, dx=None, dw=None, db=None, accumulate: bool = False, workspace=None,
                       stream=None):
    """Gradients of st_linear: dx [m, k] = dz W, dw [n, k] (+)= dz^T x (either: float32 or bfloat16), db [n] float32 (+)= sum of dz, where
    dz = dy act'(pre); pre, what st_linear left there, is asked for with an activation.  Beside bfloat16 operands dz keeps sixteen bits for a dx or dw
    in float32 (and wherever dy is float32), at the price of two products, and eight for one in bfloat16.  Only the outputs that are given are
    computed; x may be None without dw, w without dx.  accumulate=True adds to what dw and db hold.  x and w of one type; dy and pre of either; all in either
    order.  (The residual's gradient is dy.)  Returns (dx, dw, db)."""
    where = "st_linear_backward"
    mdy, m, n = _packed(dy, where)
    if (dx is not None and w is None) or (dw is not None and x is None):
        raise StError(ST_ERR_NULL, where)
    mx = mw = mpre = None
    k = 1
    a = b = (0, 0, 0)
    if dw is not None:
        mx, _, k = _packed(x, where)
    if dx is not None:
        mw, _, k = _packed(w, where)
        a = dx.data_ptr(), _out_matrix(dx, m, k, where), _dtype(dx, where)
    if dw is not None:
        b = dw.data_ptr(), _out_matrix(dw, n, k, where), _dtype(dw, where)
    if activation:
        mpre = _packed(pre, where)[0]
    grads = _GRADS_BYTES.pack(a[0], a[1], a[2], b[2], b[0], b[1], 0 if db is None else _float_vector(db, n, where), 1 if accumulate else 0)
    if workspace is None:
        workspace = _own(stream, lambda: new_linear_workspace(None if dw is None else x, None if dx is None else w, dy, activation))
    address, nbytes = _workspace(workspace, where)
    status = (_LIB or lib()).st_linear_backward(mx, mw, mdy, mpre, activation, grads, address, nbytes, _stream(stream))
    if status:
        raise StError(status, where)
    return dx, dw, db


# ---------------------------------------------------------------- the norm of many gradients, and clipping
class GradTensors:
    """The list that st_grad_clip works on, in a HOST array that is filled once (the tensors are kept alive with it): gradients, contiguous,
    float32 or bfloat16 in any mixture, and where the clipped ones go: outs (of the same lengths, either type), None in place."""

    def __init__(self, grads, outs=None):
        where = "GradTensors"
        grads = list(grads)
        outs = grads if outs is None else list(outs)
        if len(outs) != len(grads):
            raise StError(ST_ERR_SHAPE, where)
        if any(t is None for t in grads + outs):
            raise StError(ST_ERR_NULL, where)
        self.count, self.kept = len(grads), (grads, outs)
        self.array = (StGradTensor * max(self.count, 1))()
        read, written = [], []
        for a, g, o in zip(self.array, grads, outs):
            if g.numel() != o.numel() or not g.is_contiguous() or not o.is_contiguous():
                raise StError(ST_ERR_SHAPE, where)
            a.grad, a.out, a.n, a.grad_dtype, a.out_dtype = g.data_ptr(), o.data_ptr(), g.numel(), _dtype(g, where), _dtype(o, where)
            if a.n:
                written.append((a.out, a.out + o.nbytes))
                if a.grad != a.out or a.grad_dtype != a.out_dtype:
                    read.append((a.grad, a.grad + g.nbytes))
        # what is written is nobody else's: each result, and where it is not its own gradient every gradient too
        spans = sorted([(*s, True) for s in written] + [(*s, False) for s in read])
        end, end_written = 0, 0
        for first, behind, is_written in spans:
            if first < (end if is_written else end_written):
                raise StError(ST_ERR_ARG, where)
            end = max(end, behind)
            if is_written:
                end_written = max(end_written, behind)
        self.device = grads[0].device if grads else "cuda"
        self.on_device = all(t.is_cuda for t in grads + outs)
        self._bytes = None

    def norm_bytes(self) -> int:
        """Bytes of scratch that the norm of this list asks for."""
        if self._bytes is None:
            self._bytes = lib().st_grad_clip_workspace(self.array, self.count)
        return self._bytes


def new_grad_workspace(tensors: GradTensors):
    """Scratch for st_grad_clip of this list."""
    return _scratch(tensors.norm_bytes(), tensors.device, "new_grad_workspace")


def st_grad_clip(tensors: GradTensors, max_norm: float = 0.0, grad_scale: float = 1.0, grad_norm=None, workspace=None, stream=None):
    """Every gradient of the list times grad_scale, and, where the 2-norm of all of them is above max_norm > 0, times max_norm / norm, into its
    place in the list's outs.  grad_norm (float32 [1]) receives the norm before clipping.  A norm that is not finite clips nothing; one that is but passes
    float32's range clips, and grad_norm is infinite in either case."""
    where = "st_grad_clip"
    if not tensors.on_device:
        raise StError(ST_ERR_ARG, where)
    if workspace is None:
        workspace = _own(stream, lambda: new_grad_workspace(tensors))
    _check((_LIB or lib()).st_grad_clip(tensors.array, tensors.count, grad_scale, max_norm,
                                        None if grad_norm is None else _float_vector(grad_norm, 1, where),
                                        _given(workspace, tensors.norm_bytes(), where), _stream(stream)), where)


def st_graph_cache_clear():
    lib().st_graph_cache_clear()


def st_graph_cache_size() -> int:
    return int(lib().st_graph_cache_size())


def st_metric_polling(on: bool):
    lib().st_metric_polling(1 if on else 0)


def st_profile_enable(on: bool):
    lib().st_profile_enable(1 if on else 0)


def st_profile_filter(substring):
    lib().st_profile_filter(None if substring is None else substring.encode())


def st_profile_reset():
    lib().st_profile_reset()


def st_profile_read(max_stats: int = 64) -> dict:
    arr = (StKernelStat * max_stats)()
    n = lib().st_profile_read(arr, max_stats)
    if n < 0:
        raise StError(n, "st_profile_read")
    return {arr[i].name.decode(): (int(arr[i].launches), float(arr[i].total_ms)) for i in range(n)}


def st_next_stride(stride, metric, threshold, min_stride, max_stride) -> float:
    return float(lib().st_next_stride(stride, metric, threshold, min_stride, max_stride))


def st_schedule_bounds(**params) -> dict:
    """Keyword arguments: the fields of st_schedule_params.  Returns the six bounds."""
    p = StScheduleParams(**{k: float(v) for k, v in params.items()})
    out = StScheduleBounds()
    _check(lib().st_schedule_bounds(C.byref(p), C.byref(out)), "st_schedule_bounds")
    return {k: getattr(out, k) for k, _ in StScheduleBounds._fields_}


def st_schedule_total_time(n_frames, n_distill_steps, n_key_frames, t_c, **params) -> float:
    p = StScheduleParams(**{k: float(v) for k, v in params.items()})
    return float(lib().st_schedule_total_time(C.byref(p), n_frames, n_distill_steps, n_key_frames, t_c))


def st_version() -> str:
    return lib().st_version().decode()
