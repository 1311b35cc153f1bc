"""Thin ctypes binding of libchn (argument marshalling only; every step runs in the HIP kernels).

Functions carry the names of the C entry points in ``include/chn.h`` without the ``chn_`` prefix.
Arrays are ``torch.Tensor`` objects on the GPU: PyTorch supplies device memory and the stream, nothing
else.  Each call turns its tensors into ``chn_array`` descriptors (data pointer, shape, BYTE strides,
dtype), passes ``torch.cuda.current_stream()`` and raises :class:`ChnError` on a non-zero status.
The library must have been built (``python -m paper_1908_00213_amd.build``); there is no fallback.
"""
import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libchn.so")
MAX_NDIM = 8

F32, BF16, I32, I64 = 0, 1, 2, 3
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.int32: I32, torch.int64: I64}

OPS = ["copy", "add", "sub", "mul", "mad", "mad_relu", "relu", "relu_bwd", "gelu", "gelu_bwd",
       "scale", "axpy", "add_relu", "add_gelu", "fill", "sigmoid", "tanh", "sqrt", "exp", "gelu_bwd2"]
OP = {n: i for i, n in enumerate(OPS)}
REDUCE = {"sum": 0, "max": 1}
EPILOGUES = ["none", "bias", "bias_relu", "bias_gelu", "relu_bwd", "gelu_bwd", "bf16_copy"]
EPI = {n: i for i, n in enumerate(EPILOGUES)}
SCAN_KINDS = ["sigmoid", "decay"]
SCAN = {n: i for i, n in enumerate(SCAN_KINDS)}

EXPORTS = ["chn_elementwise_broadcast", "chn_reduce_axis_workspace_bytes", "chn_reduce_axis", "chn_reduce_axis_static", "chn_argmax_axis",
           "chn_gemm_workspace_bytes", "chn_gemm", "chn_linear_bwd_workspace_bytes", "chn_linear_bwd", "chn_linear_bwd_plan", "chn_lstm_fwd", "chn_lstm_bwd", "chn_lstm_step_fwd", "chn_lstm_step_bwd",
           "chn_lstm_seq_workspace_bytes", "chn_lstm_seq_supported", "chn_lstm_seq_fwd",
           "chn_lstm_seq_bwd_supported", "chn_lstm_seq_bwd_in_xcd", "chn_lstm_seq_bwd_workspace_bytes", "chn_lstm_seq_bwd", "chn_lstm_seq_spin_limit", "chn_lstm_seq_meeting",
           "chn_softmax_ce_workspace_bytes", "chn_softmax_ce_fwd", "chn_softmax_ce_bwd", "chn_softmax_ce_bwd2", "chn_softmax_ce_fwd_bwd",
           "chn_sgd_update", "chn_sgd_update_multi", "chn_adam_update_multi", "chn_embed_fwd", "chn_embed_bwd",
           "chn_dropout", "chn_rng_advance", "chn_layer_norm_fwd", "chn_layer_norm_bwd_workspace_bytes", "chn_layer_norm_bwd",
           "chn_residual_norm_fwd", "chn_residual_norm_bwd", "chn_sample_workspace_bytes", "chn_sample", "chn_logits_adjust",
           "chn_gated_scan_states", "chn_gated_scan_workspace_bytes", "chn_gated_scan_fwd", "chn_gated_scan_bwd",
           "chn_embed_scaled_fwd", "chn_embed_sorted_workspace_bytes", "chn_embed_sorted_bwd",
           "chn_status_string", "chn_last_error", "chn_version", "chn_elementwise_plan", "chn_gemm_plan", "chn_gemm_plan_kernel", "chn_gemm_plan_override",
           "chn_user_kernel_config", "chn_user_kernel_stats", "chn_user_kernel_destroy",
           "chn_elementwise_kernel_create", "chn_elementwise_kernel_prepare", "chn_elementwise_kernel_launch",
           "chn_reduction_kernel_create", "chn_reduction_kernel_workspace_bytes", "chn_reduction_kernel_prepare",
           "chn_reduction_kernel_launch", "chn_user_kernel_source"]
AXIS_ALL = -1000


def _axis_code(axis, ndim):
    """The C ABI's axis argument: one axis, CHN_AXIS_ALL for None, CHN_AXES(mask) for a tuple."""
    if axis is None:
        return AXIS_ALL
    if isinstance(axis, (tuple, list)):
        mask = 0
        for a in axis:
            mask |= 1 << (a % ndim)
        return 0x40000000 + mask
    return int(axis)


class ChnArray(C.Structure):
    _fields_ = [("data", C.c_void_p), ("ndim", C.c_int32), ("shape", C.c_int64 * MAX_NDIM),
                ("strides", C.c_int64 * MAX_NDIM), ("dtype", C.c_int32)]


class ChnError(RuntimeError):
    def __init__(self, status, detail):
        super().__init__("chn status %d: %s" % (status, detail))
        self.status = status


_lib = None


def lib():
    """Load libchn.so; fails loudly when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libchn.so is missing: run `python -m paper_1908_00213_amd.build` "
                          "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    AP = C.c_void_p                    # a reference (`_arg`): as a pointer to ChnArray by type it costs 50 ns more for each array of a call
    APP = C.POINTER(C.POINTER(ChnArray))
    vp, st = C.c_void_p, C.c_void_p
    L.chn_elementwise_broadcast.argtypes = [C.c_int, C.c_int, APP, AP, C.POINTER(C.c_float), C.c_int, st]
    L.chn_elementwise_plan.argtypes = [C.c_int, C.c_int, APP, AP]
    L.chn_reduce_axis_workspace_bytes.argtypes = [AP, C.c_int]
    L.chn_reduce_axis_workspace_bytes.restype = C.c_size_t
    L.chn_reduce_axis.argtypes = [C.c_int, AP, C.c_int, C.c_int, AP, vp, C.c_size_t, st]
    L.chn_reduce_axis_static.argtypes = [C.c_int, AP, C.c_int, C.c_int, AP, st]
    L.chn_argmax_axis.argtypes = [AP, C.c_int, C.c_int, AP, st]
    L.chn_gemm_workspace_bytes.argtypes = [AP, AP, AP]
    L.chn_gemm_workspace_bytes.restype = C.c_size_t
    L.chn_gemm_plan.argtypes = [AP, AP, AP, C.c_int]
    L.chn_gemm_plan_kernel.argtypes = [AP, AP, AP, C.c_int]
    L.chn_gemm_plan_override.argtypes = [C.c_int, C.c_int, C.c_int]
    L.chn_gemm_plan_override.restype = None
    L.chn_linear_bwd_workspace_bytes.argtypes = [AP] * 5
    L.chn_linear_bwd_workspace_bytes.restype = C.c_size_t
    L.chn_linear_bwd_plan.argtypes = [AP] * 5
    L.chn_linear_bwd.argtypes = [AP, AP, AP, C.c_int, AP, AP, AP, AP, vp, C.c_size_t, st]
    L.chn_gemm.argtypes = [AP, AP, AP, C.c_float, C.c_float, C.c_int, AP, AP, AP, vp, C.c_size_t, st]
    L.chn_lstm_fwd.argtypes = [AP, AP, AP, AP, AP, AP, st]
    L.chn_lstm_bwd.argtypes = [AP, AP, AP, AP, AP, AP, AP, st]
    L.chn_lstm_step_fwd.argtypes = [AP, AP, AP, AP, AP, AP, AP, AP, st]
    L.chn_lstm_step_bwd.argtypes = [AP, AP, AP, AP, AP, AP, AP, AP, AP, st]
    L.chn_lstm_seq_workspace_bytes.argtypes = [C.c_int64]
    L.chn_lstm_seq_workspace_bytes.restype = C.c_size_t
    L.chn_lstm_seq_supported.argtypes = [C.c_int64, C.c_int64, C.c_int]
    L.chn_lstm_seq_fwd.argtypes = [AP, AP, AP, AP, AP, AP, C.c_int64, C.c_void_p, C.c_size_t, st]
    L.chn_lstm_seq_bwd_supported.argtypes = [C.c_int64, C.c_int64, C.c_int]
    L.chn_lstm_seq_bwd_in_xcd.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_int]
    L.chn_lstm_seq_bwd_workspace_bytes.argtypes = [C.c_int64, C.c_int64]
    L.chn_lstm_seq_bwd_workspace_bytes.restype = C.c_size_t
    L.chn_lstm_seq_bwd.argtypes = [AP, AP, AP, AP, AP, AP, AP, C.c_int64, C.c_void_p, C.c_size_t, st]
    L.chn_lstm_seq_spin_limit.argtypes = [C.c_int64]
    L.chn_lstm_seq_spin_limit.restype = None
    L.chn_lstm_seq_meeting.argtypes = [C.c_int64, C.c_int]
    L.chn_lstm_seq_meeting.restype = None
    L.chn_softmax_ce_workspace_bytes.argtypes = [C.c_int64]
    L.chn_softmax_ce_workspace_bytes.restype = C.c_size_t
    L.chn_softmax_ce_fwd.argtypes = [AP, AP, C.c_int64, AP, AP, AP, vp, C.c_size_t, st]
    L.chn_softmax_ce_bwd.argtypes = [AP, AP, C.c_int64, AP, C.c_float, AP, vp, C.c_size_t, st]
    L.chn_softmax_ce_fwd_bwd.argtypes = [AP, AP, C.c_int64, AP, AP, C.c_float, AP, vp, C.c_size_t, st]
    L.chn_softmax_ce_bwd2.argtypes = [AP, AP, C.c_int64, AP, C.c_float, AP, AP, AP, vp, C.c_size_t, st]
    L.chn_sgd_update.argtypes = [AP, AP, C.c_float, AP, st]
    L.chn_sgd_update_multi.argtypes = [C.c_int, APP, APP, C.c_float, APP, st]
    L.chn_adam_update_multi.argtypes = [C.c_int, APP, APP, APP, APP, C.c_double, C.c_double, C.c_double, C.c_double, C.c_int64, APP, st]
    L.chn_embed_fwd.argtypes = [AP, AP, AP, st]
    L.chn_embed_bwd.argtypes = [AP, AP, AP, C.c_int, st]
    L.chn_dropout.argtypes = [AP, AP, C.c_double, AP, C.c_int64, AP, st]
    L.chn_rng_advance.argtypes = [AP, C.c_int64, st]
    L.chn_layer_norm_fwd.argtypes = [AP, AP, AP, C.c_double, AP, AP, AP, st]
    L.chn_layer_norm_bwd_workspace_bytes.argtypes = [AP]
    L.chn_layer_norm_bwd_workspace_bytes.restype = C.c_size_t
    L.chn_layer_norm_bwd.argtypes = [AP] * 8 + [vp, C.c_size_t, st]
    L.chn_residual_norm_fwd.argtypes = [AP, AP, C.c_double, AP, C.c_int64, AP, AP, C.c_double, AP, AP, AP, AP, st]
    L.chn_residual_norm_bwd.argtypes = [AP] * 6 + [C.c_double, AP, C.c_int64, AP, AP, AP, AP, vp, C.c_size_t, st]
    L.chn_sample_workspace_bytes.argtypes = [AP]
    L.chn_sample_workspace_bytes.restype = C.c_size_t
    L.chn_sample.argtypes = [AP] * 7 + [vp, C.c_size_t, st]
    L.chn_logits_adjust.argtypes = [AP] * 11 + [st]
    L.chn_gated_scan_states.argtypes = [C.c_int64]
    L.chn_gated_scan_states.restype = C.c_int64
    L.chn_gated_scan_workspace_bytes.argtypes = [AP]
    L.chn_gated_scan_workspace_bytes.restype = C.c_size_t
    L.chn_gated_scan_fwd.argtypes = [C.c_int] + [AP] * 7 + [vp, C.c_size_t, st]
    L.chn_gated_scan_bwd.argtypes = [C.c_int] + [AP] * 9 + [vp, C.c_size_t, st]
    L.chn_embed_scaled_fwd.argtypes = [AP, AP, C.c_double, AP, st]
    L.chn_embed_sorted_workspace_bytes.argtypes = [AP, AP]
    L.chn_embed_sorted_workspace_bytes.restype = C.c_size_t
    L.chn_embed_sorted_bwd.argtypes = [AP, AP, C.c_double, AP, C.c_int, vp, C.c_size_t, st]
    L.chn_status_string.argtypes = [C.c_int32]
    L.chn_status_string.restype = C.c_char_p
    L.chn_last_error.argtypes = []
    L.chn_last_error.restype = C.c_char_p
    L.chn_version.argtypes = []
    cs, KP, dp = C.c_char_p, C.c_void_p, C.POINTER(C.c_double)
    L.chn_user_kernel_config.argtypes = [cs, cs]
    L.chn_user_kernel_stats.argtypes = [C.POINTER(C.c_longlong)] * 3
    L.chn_user_kernel_stats.restype = None
    L.chn_user_kernel_destroy.argtypes = [KP]
    L.chn_user_kernel_destroy.restype = None
    L.chn_elementwise_kernel_create.argtypes = [cs, cs, cs, cs, cs, C.POINTER(KP)]
    L.chn_elementwise_kernel_prepare.argtypes = [KP, C.c_int, APP, C.c_int, APP]
    L.chn_elementwise_kernel_launch.argtypes = [KP, C.c_int, APP, C.c_int, APP, dp, st]
    L.chn_reduction_kernel_create.argtypes = [cs, cs, cs, cs, cs, cs, cs, cs, C.POINTER(KP)]
    L.chn_reduction_kernel_workspace_bytes.argtypes = [KP, C.c_int, APP, C.c_int, APP, C.c_int, C.c_int]
    L.chn_reduction_kernel_workspace_bytes.restype = C.c_size_t
    L.chn_reduction_kernel_prepare.argtypes = [KP, C.c_int, APP, C.c_int, APP, C.c_int, C.c_int]
    L.chn_reduction_kernel_launch.argtypes = [KP, C.c_int, APP, C.c_int, APP, dp, C.c_int, C.c_int, vp, C.c_size_t, st]
    L.chn_user_kernel_source.argtypes = [KP, C.c_int, APP, C.c_int, APP, C.c_int, C.c_int, C.c_char_p, C.c_size_t,
                                         C.POINTER(C.c_size_t)]
    for name in EXPORTS:
        fn = getattr(L, name)
        if fn.restype is C.c_int and name not in ("chn_version", "chn_elementwise_plan", "chn_gemm_plan", "chn_gemm_plan_kernel", "chn_linear_bwd_plan"):  # i.e. not set above
            fn.restype = C.c_int32
    _lib = L
    return L


class _Kept:
    """A tensor's descriptor, with the reference to it that calls take and what shows whether it still holds: the tensor's address, which another storage
    changes, and its version, which every operation in place changes.  A tensor that is copied or pickled carries nothing in its place."""
    __slots__ = ("ref", "ptr", "version", "device", "desc", "pointer", "shape", "strides")

    def __reduce__(self):
        return set, ()

    def __deepcopy__(self, memo):
        return None


# By dtype: the descriptor's code and the element's bytes; by the number of dimensions: a descriptor's fields, which are written in one go.
_ELEMENTS = {t: (code, torch.empty(0, dtype=t).element_size()) for t, code in _DTYPES.items()}
_FIELDS = [struct.Struct("@Pi4x%dq%dx%dq%dxi4x" % (n, 8 * (MAX_NDIM - n), n, 8 * (MAX_NDIM - n))) for n in range(MAX_NDIM + 1)]
assert all(f.size == C.sizeof(ChnArray) for f in _FIELDS)


def _describe(t):
    """The descriptor of a tensor, kept on it from here on: parameters, inputs and gradients are described thousands of times."""
    k = _Kept()
    k.desc = a = ChnArray()
    k.shape = shape = t.shape
    k.strides = strides = t.stride()
    k.ptr = ptr = t.data_ptr()
    code, size = _ELEMENTS[t.dtype]
    n = len(shape)
    _FIELDS[n].pack_into(a, 0, ptr, n, *shape, *[s * size for s in strides], code)
    k.ref, k.pointer, k.device = C.byref(a), None, None      # (the latter two when they are asked for)
    try:
        k.version = t._version
    except RuntimeError:                                 # (not counted in inference mode)
        k.version = None
    t._chn_kept = k
    return k


def _again(t):
    """What is kept on a tensor of which nothing is known yet, or whose address or version is another one: made anew where more has changed than what it holds."""
    k = getattr(t, "_chn_kept", None)
    if type(k) is not _Kept or k.ptr != t.data_ptr() or k.shape != t.shape or k.strides != t.stride():
        return _describe(t)
    version = None if t.is_inference() else t._version
    if version == k.version:
        return k
    same = _Kept()                                       # (the old one may be kept on a shallow copy too)
    same.ref, same.ptr, same.version, same.device, same.desc = k.ref, k.ptr, version, k.device, k.desc
    same.pointer, same.shape, same.strides = k.pointer, k.shape, k.strides
    t._chn_kept = same
    return same


def _kept(t):
    """The descriptor of a tensor, as it is now: after resize_, set_, transpose_, an `out=` that resized it, an assignment to .data.  (Only an assignment to .data of
    another view of the very same memory shows nowhere.)"""
    try:
        k = t._chn_kept
        if k.ptr == t.data_ptr() and k.version == t._version:
            return k
    except (AttributeError, RuntimeError):               # (none yet, or what a copied tensor carries; a version that is not counted)
        pass
    return _again(t)


def desc(t):
    """chn_array descriptor of a tensor (or None).  It holds as long as the tensor is not given other memory or another shape."""
    if t is None or type(t) is ChnArray:
        return t
    return _kept(t).desc


def _arg(t):
    """A call's argument for a tensor, a descriptor or None."""
    if t is None:
        return None
    return C.byref(t) if type(t) is ChnArray else _kept(t).ref


_HANDLES = {}                      # streams' handles as calls take them


def _here(stream, *arrays):
    """For `_raw` calls: references to the descriptors of arrays, which have to lie on the current device (of a descriptor that is not known), and behind them the handle of
    the stream, None: torch's current one.  (A call with twelve arrays spends more time on these than on its launch.)"""
    current = _raw_device() if _raw_device is not None else torch.cuda.current_device()
    try:
        out = [None if t is None else k.ref if (k := t._chn_kept).ptr == t.data_ptr() and k.version == t._version and k.device == current else _look(t, current)
               for t in arrays]
    except (AttributeError, RuntimeError):
        out = [None if t is None else _look(t, current) for t in arrays]
    if stream is None:
        raw = _raw_stream(current) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream
        stream = _HANDLES.get(raw)
        if stream is None:
            if len(_HANDLES) >= 256:
                _HANDLES.clear()
            stream = _HANDLES[raw] = C.c_void_p(raw)
    elif not isinstance(stream, C.c_void_p):
        stream = C.c_void_p(stream)
    out.append(stream)
    return out


def _look(t, current):
    if type(t) is ChnArray:
        return C.byref(t)
    k = _kept(t)
    if k.device is None:
        k.device = t.get_device()
    if k.device != current:
        raise ValueError("an array lies on %s, the current device is cuda:%d" % ("the host" if k.device < 0 else "cuda:%d" % k.device, current))
    return k.ref


class _RawCalls(dict):
    """The entry points without argument types, whose conversions cost half a microsecond a call: they are given references, ctypes numbers and None only."""

    def __missing__(self, name):
        f = self[name] = lib()[name]
        f.restype = C.c_int32
        return f


_raw = _RawCalls()


def raw_desc(ptr, shape, strides_bytes, dtype):
    """Descriptor from raw fields (used by tests of the validation paths)."""
    a = ChnArray()
    a.data = ptr
    a.ndim = len(shape)
    for d, (n, s) in enumerate(zip(shape, strides_bytes)):
        if d < MAX_NDIM:
            a.shape[d] = n
            a.strides[d] = s
    a.dtype = dtype
    return a


def _ref(a):
    return None if a is None else C.byref(a)


_POINTER_ARRAYS = {}               # by length


def _ptrs(arrays):
    """Pointers to the descriptors of tensors, or to descriptors; NULL for None."""
    n = len(arrays)
    make = _POINTER_ARRAYS.get(n)
    if make is None:
        make = _POINTER_ARRAYS[n] = C.POINTER(ChnArray) * max(1, n)
    arr = make()
    for i, t in enumerate(arrays):
        if t is not None:
            if type(t) is ChnArray:
                arr[i] = C.pointer(t)
                continue
            k = _kept(t)
            if k.pointer is None:
                k.pointer = C.pointer(k.desc)
            arr[i] = k.pointer
    return arr


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    """hipStream_t of torch's current stream (the raw-handle query costs a fraction of a microsecond,
    the Stream object several)."""
    if _raw_stream is not None and _raw_device is not None:
        return C.c_void_p(_raw_stream(_raw_device()))
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(status):
    if status != 0:
        L = lib()
        raise ChnError(status, "%s: %s" % (L.chn_status_string(status).decode(), L.chn_last_error().decode()))


def _ws(t):
    if t is None:
        return None, 0
    return C.c_void_p(t.data_ptr()), t.numel() * t.element_size()


_NO_BYTES = C.c_size_t(0)


def _ws_here(t):
    """The same for `_raw` calls whose arrays have to lie on the current device."""
    if t is None:
        return None, _NO_BYTES
    if t.get_device() != (_raw_device() if _raw_device is not None else torch.cuda.current_device()):
        raise ValueError("the workspace does not lie on the current device")
    return C.c_void_p(t.data_ptr()), C.c_size_t(t.nbytes)


def version():
    return lib().chn_version()


def elementwise_plan(op, inputs, out):
    return lib().chn_elementwise_plan(OP[op] if isinstance(op, str) else op, len(inputs), _ptrs(inputs), _arg(out))


def elementwise_broadcast(op, inputs, out, scalars=(), stream=None):
    sc = (C.c_float * max(1, len(scalars)))(*[float(s) for s in scalars])
    _check(lib().chn_elementwise_broadcast(OP[op] if isinstance(op, str) else op, len(inputs), _ptrs(inputs),
                                           _arg(out), sc, len(scalars),
                                           _stream() if stream is None else stream))
    return out


def cast(x, dtype):
    """A copy of `x` in another storage type through the library's own kernel (CHN_OP_COPY: fp32 values
    round to nearest even on their way to bfloat16); torch only allocates the result."""
    if x.dtype == dtype:
        return x
    return elementwise_broadcast("copy", [x], torch.empty(x.shape, dtype=dtype, device=x.device))


def reduce_axis_workspace_bytes(x, axis):
    d = desc(x)
    return lib().chn_reduce_axis_workspace_bytes(_ref(d), _axis_code(axis, d.ndim))


def reduce_axis(op, x, axis, out, keepdims=False, ws=None, stream=None):
    """axis: an int, a tuple of ints (several axes at once) or None (all of them)."""
    p, n = _ws(ws)
    axis = _axis_code(axis, desc(x).ndim)
    _check(lib().chn_reduce_axis(REDUCE[op] if isinstance(op, str) else op, _arg(x), axis,
                                 int(keepdims), _arg(out), p, n,
                                 _stream() if stream is None else stream))
    return out


def reduce_axis_static(op, x, axis, out, keepdims=False, stream=None):
    """reduce_axis without a workspace argument and without any allocation (partial sums in the
    library's built-in per-device array)."""
    axis = _axis_code(axis, desc(x).ndim)
    _check(lib().chn_reduce_axis_static(REDUCE[op] if isinstance(op, str) else op, _arg(x), axis,
                                        int(keepdims), _arg(out), _stream() if stream is None else stream))
    return out


def argmax_axis(x, axis, out, keepdims=False, stream=None):
    _check(lib().chn_argmax_axis(_arg(x), int(axis), int(keepdims), _arg(out),
                                 _stream() if stream is None else stream))
    return out


def gemm_workspace_bytes(A, B, Cm):
    return lib().chn_gemm_workspace_bytes(_arg(A), _arg(B), _arg(Cm))


def gemm_plan(A, B, Cm, have_workspace=False):
    """(tile, direct_copy, splits) chn_gemm would use: tile 0/1/2 = 64/128/256 square, 3 = 256 x 128."""
    code = lib().chn_gemm_plan(_arg(A), _arg(B), _arg(Cm), 1 if have_workspace else 0)
    if code < 0:
        _check(code)
    return code & 3, bool(code & 4), code >> 4


def gemm_plan_eight_waves(A, B, Cm, have_workspace=False):
    """Whether the plain product would run on the eight-wave form of the direct-copy kernel (bf16) or on the
    three-part kernel (fp32)."""
    code = lib().chn_gemm_plan(_arg(A), _arg(B), _arg(Cm), 1 if have_workspace else 0)
    if code < 0:
        _check(code)
    return bool(code & 8)


GEMM_KERNELS = ("staged", "direct4", "direct8", "parts", "small")


def gemm_plan_kernel(A, B, Cm, have_workspace=False):
    """The kernel the plain product would run on, one of GEMM_KERNELS."""
    code = lib().chn_gemm_plan_kernel(_arg(A), _arg(B), _arg(Cm), 1 if have_workspace else 0)
    if code < 0:
        _check(code)
    return GEMM_KERNELS[code]


def gemm_plan_override(tile=-1, splits=-1, direct_copy=-1):
    """Test hook: force the macro tile / K splits / keep products off the direct-copy kernel (-1: planner's choice)."""
    lib().chn_gemm_plan_override(int(tile), int(splits), int(direct_copy))


def gemm(A, B, Cm, alpha=1.0, beta=0.0, epilogue="none", bias=None, aux=None, preact_out=None,
         ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().chn_gemm(_arg(A), _arg(B), _arg(Cm), float(alpha), float(beta),
                          EPI[epilogue] if isinstance(epilogue, str) else epilogue,
                          _arg(bias), _arg(aux), _arg(preact_out), p, n,
                          _stream() if stream is None else stream))
    return Cm


def linear_bwd_workspace_bytes(dv, W, x, dx, dW):
    return lib().chn_linear_bwd_workspace_bytes(_arg(dv), _arg(W), _arg(x), _arg(dx), _arg(dW))


def linear_bwd_in_one_launch(dv, W, x, dx, dW):
    """Whether linear_bwd would be one kernel (outputs apart from the other arrays)."""
    code = lib().chn_linear_bwd_plan(_arg(dv), _arg(W), _arg(x), _arg(dx), _arg(dW))
    if code < 0:
        _check(code)
    return bool(code)


def linear_bwd(dv, W, x, dW, db=None, dx=None, epilogue="none", aux=None, ws=None, stream=None):
    """dW = dv^T x, db = column sums of dv, dx = epilogue(dv W): the backward of y = x W^T + b."""
    p, n = _ws(ws)
    _check(lib().chn_linear_bwd(_arg(dv), _arg(W), _arg(x), EPI[epilogue] if isinstance(epilogue, str) else epilogue,
                                _arg(aux), _arg(dx), _arg(dW), _arg(db), p, n,
                                _stream() if stream is None else stream))


def lstm_fwd(z, bias, c_prev, c, h, gates=None, stream=None):
    _check(lib().chn_lstm_fwd(_arg(z), _arg(bias), _arg(c_prev), _arg(c),
                              _arg(h), _arg(gates), _stream() if stream is None else stream))


def lstm_bwd(gates, c_prev, c, dh, dc_next, dz, dc_prev, stream=None):
    _check(lib().chn_lstm_bwd(_arg(gates), _arg(c_prev), _arg(c), _arg(dh),
                              _arg(dc_next), _arg(dz), _arg(dc_prev),
                              _stream() if stream is None else stream))


def lstm_step_fwd(zx, h_prev, Ut, bias, c_prev, c, h, gates=None, stream=None):
    _check(lib().chn_lstm_step_fwd(_arg(zx), _arg(h_prev), _arg(Ut), _arg(bias), _arg(c_prev),
                                   _arg(c), _arg(h), _arg(gates), _stream() if stream is None else stream))


def lstm_step_bwd(dz_next, U, dh, gates, c_prev, c, dc_next, dz, dc_prev, stream=None):
    _check(lib().chn_lstm_step_bwd(_arg(dz_next), _arg(U), _arg(dh), _arg(gates), _arg(c_prev),
                                   _arg(c), _arg(dc_next), _arg(dz), _arg(dc_prev),
                                   _stream() if stream is None else stream))


def lstm_seq_workspace_bytes(batch):
    return lib().chn_lstm_seq_workspace_bytes(int(batch))


def lstm_seq_supported(batch, hidden, dtype):
    """Whether lstm_seq_fwd takes this batch and hidden width (torch dtype) on the current device."""
    return lib().chn_lstm_seq_supported(int(batch), int(hidden), _DTYPES[dtype]) == 0


def lstm_seq_status(ws):
    """The status word lstm_seq_fwd left in its workspace (synchronises): 0 = complete, 1 = a wait ran out."""
    return int(ws[:4].view(torch.int32).item())


def lstm_seq_fwd(zx, Ut, bias, Hs, Cs, gates, n_steps, ws, stream=None):
    """All n_steps forward steps in one launch.  ws[0:4] reads 1 after synchronisation if a wait ran out."""
    p, n = _ws(ws)
    _check(lib().chn_lstm_seq_fwd(_arg(zx), _arg(Ut), _arg(bias), _arg(Hs), _arg(Cs),
                                  _arg(gates), int(n_steps), p, n, _stream() if stream is None else stream))


def lstm_seq_bwd_supported(batch, hidden, dtype):
    return lib().chn_lstm_seq_bwd_supported(int(batch), int(hidden), _DTYPES[dtype]) == 0


def lstm_seq_bwd_in_xcd(batch, hidden, n_steps, dtype):
    """Whether lstm_seq_bwd walks these sizes inside the XCDs of the current device: then it is the faster one in bfloat16 too (128 x 672: 3.8 us per
    step, the fused per-step call 11.5, the kernel that exchanges through device memory 11.9)."""
    return lib().chn_lstm_seq_bwd_in_xcd(int(batch), int(hidden), int(n_steps), _DTYPES[dtype]) == 1


def lstm_seq_bwd_workspace_bytes(batch, hidden):
    return lib().chn_lstm_seq_bwd_workspace_bytes(int(batch), int(hidden))


def lstm_seq_bwd(U, dHs, gates, Cs, dc_last, dZ, dc0, n_steps, ws, stream=None):
    """Back-propagation through all n_steps steps in one launch; status word in ws as for lstm_seq_fwd."""
    p, n = _ws(ws)
    _check(lib().chn_lstm_seq_bwd(_arg(U), _arg(dHs), _arg(gates), _arg(Cs), _arg(dc_last),
                                  _arg(dZ), _arg(dc0), int(n_steps), p, n, _stream() if stream is None else stream))


def lstm_seq_spin_limit(polls):
    lib().chn_lstm_seq_spin_limit(int(polls))


def lstm_seq_meeting(patience=-1, share_l2=True):
    lib().chn_lstm_seq_meeting(int(patience), int(share_l2))


def softmax_ce_workspace_bytes(n_rows):
    return lib().chn_softmax_ce_workspace_bytes(int(n_rows))


def softmax_ce_fwd(logits, labels, loss_mean, loss_rows=None, lse=None, ignore_label=-1, ws=None,
                   stream=None):
    p, n = _ws(ws)
    _check(lib().chn_softmax_ce_fwd(_arg(logits), _arg(labels), int(ignore_label),
                                    _arg(loss_mean), _arg(loss_rows), _arg(lse), p, n,
                                    _stream() if stream is None else stream))
    return loss_mean


def softmax_ce_bwd(logits, labels, dlogits, lse=None, upstream=1.0, ignore_label=-1, ws=None,
                   stream=None):
    p, n = _ws(ws)
    _check(lib().chn_softmax_ce_bwd(_arg(logits), _arg(labels), int(ignore_label),
                                    _arg(lse), float(upstream), _arg(dlogits), p, n,
                                    _stream() if stream is None else stream))
    return dlogits


def softmax_ce_bwd2(logits, labels, gg, dlogits, dupstream=None, lse=None, upstream=1.0, ignore_label=-1, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().chn_softmax_ce_bwd2(_arg(logits), _arg(labels), int(ignore_label), _arg(lse), float(upstream),
                                     _arg(gg), _arg(dlogits), _arg(dupstream), p, n,
                                     _stream() if stream is None else stream))
    return dlogits


def softmax_ce_fwd_bwd(logits, labels, loss_mean, dlogits, lse=None, upstream=1.0, ignore_label=-1, ws=None,
                       stream=None):
    p, n = _ws(ws)
    _check(lib().chn_softmax_ce_fwd_bwd(_arg(logits), _arg(labels), int(ignore_label), _arg(loss_mean),
                                        _arg(lse), float(upstream), _arg(dlogits), p, n,
                                        _stream() if stream is None else stream))
    return loss_mean


def sgd_update(param, grad, lr, lowp_copy=None, stream=None):
    _check(lib().chn_sgd_update(_arg(param), _arg(grad), float(lr), _arg(lowp_copy),
                                _stream() if stream is None else stream))


def sgd_update_multi(params, grads, lr, lowp_copies=None, stream=None):
    _check(lib().chn_sgd_update_multi(len(params), _ptrs(params), _ptrs(grads), float(lr),
                                      None if lowp_copies is None else _ptrs(lowp_copies),
                                      _stream() if stream is None else stream))


def _row_block(t, rows):
    """Descriptor of the first `rows` rows of a 2-d tensor and the byte distance to the next such block:
    a sequence of calls over consecutive row blocks moves the data pointer instead of slicing."""
    isz = t.element_size()
    return raw_desc(t.data_ptr(), (rows, t.shape[1]), (t.stride(0) * isz, t.stride(1) * isz), _DTYPES[t.dtype]), rows * t.stride(0) * isz


def lstm_step_fwd_seq(zx, Hs, Ut, bias, Cs, gates, n_steps, stream=None):
    """n_steps calls of lstm_step_fwd over time-major buffers: step t reads rows t*B.. of zx, block t of
    Hs and Cs ((n_steps+1)*B rows, block 0 = initial state) and writes block t+1 of Hs and Cs and block t
    of gates.  Same calls as the loop over slices; only the marshalling is done once."""
    L, st = lib(), (_stream() if stream is None else stream)
    Bn = zx.shape[0] // n_steps
    if zx.shape[0] != n_steps * Bn or Hs.shape[0] != (n_steps + 1) * Bn or Cs.shape[0] != (n_steps + 1) * Bn or gates.shape[0] != n_steps * Bn:
        raise ValueError("lstm_step_fwd_seq: buffers do not hold %d steps" % n_steps)
    (zd, zs), (hp, hs), (cp, cs), (gd, gs) = _row_block(zx, Bn), _row_block(Hs, Bn), _row_block(Cs, Bn), _row_block(gates, Bn)
    (hn, _), (cn, _) = _row_block(Hs, Bn), _row_block(Cs, Bn)
    hn.data += hs
    cn.data += cs
    ut, bd = _arg(Ut), _arg(bias)
    for _ in range(n_steps):
        _check(L.chn_lstm_step_fwd(C.byref(zd), C.byref(hp), ut, bd, C.byref(cp), C.byref(cn), C.byref(hn), C.byref(gd), st))
        zd.data += zs; hp.data += hs; hn.data += hs; cp.data += cs; cn.data += cs; gd.data += gs


def lstm_step_bwd_seq(dZ, U, dHs, gates, Cs, dc_last, dc, n_steps, stream=None):
    """The n_steps calls of lstm_step_bwd of one back-propagation through time, last step first: dZ, dHs
    and gates hold n_steps row blocks, Cs n_steps + 1; dc_last (or None) is the gradient reaching the
    final cell state; dc = two (B, H) buffers that take turns (the one of step 0 holds the gradient
    of the initial cell state afterwards)."""
    L, st = lib(), (_stream() if stream is None else stream)
    Bn = dZ.shape[0] // n_steps
    if dZ.shape[0] != n_steps * Bn or dHs.shape[0] != n_steps * Bn or gates.shape[0] != n_steps * Bn or Cs.shape[0] != (n_steps + 1) * Bn:
        raise ValueError("lstm_step_bwd_seq: buffers do not hold %d steps" % n_steps)
    (zd, zs), (zn, _), (hd, hs), (gd, gs), (cp, cs), (cn, _) = (_row_block(dZ, Bn), _row_block(dZ, Bn), _row_block(dHs, Bn),
                                                             _row_block(gates, Bn), _row_block(Cs, Bn), _row_block(Cs, Bn))
    last = n_steps - 1
    zd.data += last * zs; zn.data += (last + 1) * zs; hd.data += last * hs; gd.data += last * gs; cp.data += last * cs; cn.data += (last + 1) * cs
    ud = _arg(U)
    dcd = [C.byref(desc(dc[0])), C.byref(desc(dc[1]))]
    dc_next = _arg(dc_last)
    for t in range(last, -1, -1):
        _check(L.chn_lstm_step_bwd(None if t == last else C.byref(zn), ud, C.byref(hd), C.byref(gd), C.byref(cp), C.byref(cn),
                                   dc_next, C.byref(zd), dcd[t & 1], st))
        dc_next = dcd[t & 1]
        zd.data -= zs; zn.data -= zs; hd.data -= hs; gd.data -= gs; cp.data -= cs; cn.data -= cs


def adam_update_multi(params, grads, ms, vs, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, lowp_copies=None, stream=None):
    _check(lib().chn_adam_update_multi(len(params), _ptrs(params), _ptrs(grads), _ptrs(ms), _ptrs(vs), float(lr), float(beta1),
                                       float(beta2), float(eps), int(step), None if lowp_copies is None else _ptrs(lowp_copies),
                                       _stream() if stream is None else stream))


def embed_fwd(table, ids, out, stream=None):
    _check(lib().chn_embed_fwd(_arg(table), _arg(ids), _arg(out),
                               _stream() if stream is None else stream))
    return out


def embed_bwd(ids, dout, dtable, accumulate=False, stream=None):
    _check(lib().chn_embed_bwd(_arg(ids), _arg(dout), _arg(dtable), int(accumulate),
                               _stream() if stream is None else stream))
    return dtable


def dropout(x, y, ratio, rng=None, site=0, residual=None, stream=None):
    """y = (residual +) dropout(x); rng: int64 tensor (seed, offset).  The gradient of x is the same call on the gradient of y."""
    dx, dr, dg, dy, st = _here(stream, x, residual, rng, y)
    status = _raw["chn_dropout"](dx, dr, C.c_double(ratio), dg, C.c_int64(int(site)), dy, st)
    if status:
        _check(status)
    return y


def rng_advance(rng, steps=1, stream=None):
    """rng[1] += steps on the stream: later draws (a replayed graph's too) use other masks."""
    dg, st = _here(stream, rng)
    _check(_raw["chn_rng_advance"](dg, C.c_int64(int(steps)), st))
    return rng


def layer_norm_fwd(x, y, gamma=None, beta=None, eps=1e-5, mean=None, rstd=None, stream=None):
    """mean: (N,), or (N,2) with what its rounding left, which keeps the digits of the gradients of rows with a large mean."""
    dx, dg, db, dy, dm, dr, st = _here(stream, x, gamma, beta, y, mean, rstd)
    status = _raw["chn_layer_norm_fwd"](dx, dg, db, C.c_double(eps), dy, dm, dr, st)
    if status:
        _check(status)
    return y


def layer_norm_bwd_workspace_bytes(x):
    return lib().chn_layer_norm_bwd_workspace_bytes(_arg(x))


def layer_norm_bwd(dy, x, mean, rstd, dx, gamma=None, dgamma=None, dbeta=None, ws=None, stream=None):
    p, n = _ws_here(ws)
    ddy, d_x, dm, dr, dg, ddx, ddg, ddb, st = _here(stream, dy, x, mean, rstd, gamma, dx, dgamma, dbeta)
    status = _raw["chn_layer_norm_bwd"](ddy, d_x, dm, dr, dg, ddx, ddg, ddb, p, n, st)
    if status:
        _check(status)
    return dx


def residual_norm_fwd(x, residual, s, y, gamma=None, beta=None, eps=1e-5, mean=None, rstd=None, ratio=0.0, rng=None, site=0, stream=None):
    """s = residual + dropout(x), y = layer_norm(s)."""
    dx, dres, ds, dy, dg, db, dm, dr, drng, st = _here(stream, x, residual, s, y, gamma, beta, mean, rstd, rng)
    status = _raw["chn_residual_norm_fwd"](dx, dres, C.c_double(ratio), drng, C.c_int64(int(site)), dg, db, C.c_double(eps), ds, dy, dm, dr, st)
    if status:
        _check(status)
    return y


def residual_norm_bwd(dy, ds, s, mean, rstd, dresidual, dx, gamma=None, dgamma=None, dbeta=None, ratio=0.0, rng=None, site=0, ws=None, stream=None):
    """dresidual and dx from the gradients dy of y and ds of s (or None)."""
    p, n = _ws_here(ws)
    ddy, dds, d_s, dm, dr, dg, drng, ddres, ddx, ddg, ddb, st = _here(stream, dy, ds, s, mean, rstd, gamma, rng, dresidual, dx, dgamma, dbeta)
    status = _raw["chn_residual_norm_bwd"](ddy, dds, d_s, dm, dr, dg, C.c_double(ratio), drng, C.c_int64(int(site)), ddres, ddx, ddg, ddb, p, n, st)
    if status:
        _check(status)
    return dx


def sample_workspace_bytes(logits):
    return lib().chn_sample_workspace_bytes(_arg(logits))


def sample(logits, u, out, temperature=None, top_k=None, top_p=None, min_p=None, ws=None, stream=None):
    """out[n]: a token of row n, drawn by u[n]; parameters are tensors of one value for each row (stride 0: one for all), None: not used."""
    p, n = _ws_here(ws)
    dz, du, dt, dk, dp, dm, do, st = _here(stream, logits, u, temperature, top_k, top_p, min_p, out)
    status = _raw["chn_sample"](dz, du, dt, dk, dp, dm, do, p, n, st)
    if status:
        _check(status)
    return out


def logits_adjust(logits, out, tokens=None, lengths=None, prompt=None, repetition=None, frequency=None, presence=None, bias_ids=None, bias=None,
                  allowed=None, stream=None):
    """out = logits with penalties for a row's tokens, biases and a mask of allowed tokens (out may be logits); None: not used."""
    dz, dt, dl, dp, dr, df, ds, di, db, da, do, st = _here(stream, logits, tokens, lengths, prompt, repetition, frequency, presence, bias_ids, bias, allowed, out)
    status = _raw["chn_logits_adjust"](dz, dt, dl, dp, dr, df, ds, di, db, da, do, st)
    if status:
        _check(status)
    return out


def gated_scan_states_shape(steps, batch, cols):
    """Of the fp32 states that a forward pass keeps for its backward pass."""
    return lib().chn_gated_scan_states(int(steps)), int(batch), int(cols)


def gated_scan_workspace_bytes(gate):
    return lib().chn_gated_scan_workspace_bytes(_arg(gate))


def _scan_kind(kind):
    return C.c_int(SCAN[kind] if isinstance(kind, str) else kind)


def gated_scan_fwd(gate, x, y, h0=None, h_last=None, states=None, lengths=None, kind="sigmoid", ws=None, stream=None):
    """y[t] = h_t = a h_{t-1} + (1 - a) x[t], a = sigmoid(gate[t]) ("sigmoid"), or gate[t] h_{t-1} + x[t] ("decay"); (T, B, D).  states: for the backward pass."""
    p, n = _ws_here(ws)
    dg, dx, d0, dl, dy, dh, ds, st = _here(stream, gate, x, h0, lengths, y, h_last, states)
    status = _raw["chn_gated_scan_fwd"](_scan_kind(kind), dg, dx, d0, dl, dy, dh, ds, p, n, st)
    if status:
        _check(status)
    return y


def gated_scan_bwd(gate, x, states, dy, dgate, dx, dh_last=None, dh0=None, lengths=None, kind="sigmoid", ws=None, stream=None):
    """Gradients of gate, x and h0 from those of y and h_last, with the states that the forward pass kept."""
    p, n = _ws_here(ws)
    dg, d_x, ds, dl, ddy, ddh, ddg, ddx, dd0, st = _here(stream, gate, x, states, lengths, dy, dh_last, dgate, dx, dh0)
    status = _raw["chn_gated_scan_bwd"](_scan_kind(kind), dg, d_x, ds, dl, ddy, ddh, ddg, ddx, dd0, p, n, st)
    if status:
        _check(status)
    return dx


def embed_scaled_fwd(table, ids, out, scale=1.0, stream=None):
    """out[n] = scale * table[ids[n]]"""
    dt, di, do, st = _here(stream, table, ids, out)
    status = _raw["chn_embed_scaled_fwd"](dt, di, C.c_double(scale), do, st)
    if status:
        _check(status)
    return out


def embed_sorted_workspace_bytes(ids, dtable):
    return lib().chn_embed_sorted_workspace_bytes(_arg(ids), _arg(dtable))


def embed_sorted_bwd(ids, dout, dtable, scale=1.0, accumulate=False, ws=None, stream=None):
    """dtable[v] = (dtable[v] +) scale * sum of the rows of dout whose id is v, by sorting the ids."""
    p, n = _ws_here(ws)
    di, do, dt, st = _here(stream, ids, dout, dtable)
    status = _raw["chn_embed_sorted_bwd"](di, do, C.c_double(scale), dt, C.c_int(int(accumulate)), p, n, st)
    if status:
        _check(status)
    return dtable


# ---- user-defined kernels ---------------------------------------------------------------------------------
def user_kernel_config(cache_dir=None, arch=None):
    enc = lambda v: None if v is None else str(v).encode()
    _check(lib().chn_user_kernel_config(enc(cache_dir), enc(arch)))


def user_kernel_stats():
    """(compiler runs, code objects found on disk, found in memory) since the library was loaded."""
    v = [C.c_longlong(0) for _ in range(3)]
    lib().chn_user_kernel_stats(*[C.byref(x) for x in v])
    return tuple(int(x.value) for x in v)


_TORCH_OF = {F32: torch.float32, BF16: torch.bfloat16, I32: torch.int32, I64: torch.int64}
_CONCRETE = {"float32": F32, "bfloat16": BF16, "int32": I32, "int64": I64}


class _UserKernel:
    """Owner of a chn_user_kernel handle.  Arguments of a call: arrays (tensors or descriptors) and
    Python numbers for scalar parameters, inputs first, then optionally the outputs; outputs that
    are left out are allocated (shape from broadcasting, dtype from the declaration or from the
    arrays that bind the output's type parameter)."""

    def __init__(self, handle, in_params, out_params, name):
        self._h = handle
        self.name = name
        split = lambda text: [tuple(item.split()) for item in text.split(",") if item.strip()]
        self.in_params, self.out_params = split(in_params), split(out_params)

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h is not None and _lib is not None:
            _lib.chn_user_kernel_destroy(h)

    def _split(self, args):
        n_in, n_out = len(self.in_params), len(self.out_params)
        if len(args) not in (n_in, n_in + n_out):
            raise TypeError("%s takes %d inputs (and optionally %d outputs), got %d arguments"
                            % (self.name, n_in, n_out, len(args)))
        ins = list(args[:n_in])
        scalars = [float(a) for a in ins if isinstance(a, (int, float))]
        arrays = [None if isinstance(a, (int, float)) else a for a in ins]
        return arrays, scalars, list(args[n_in:])

    def _out_dtype(self, j, arrays):
        t = self.out_params[j][0]
        if t in _CONCRETE:
            return _TORCH_OF[_CONCRETE[t]]
        for (pt, _), a in zip(self.in_params, arrays):
            if pt == t and a is not None:
                return a.dtype
        raise TypeError("%s: no input binds the type parameter %s of output %s" % (self.name, t, self.out_params[j][1]))

    @staticmethod
    def _marshal(arrays, scalars):
        ds = [desc(a) for a in arrays]
        sc = (C.c_double * max(1, len(scalars)))(*scalars)
        return ds, sc

    def source(self, *args, axis=None, keepdims=False):
        """Generated source of the specialisation this call would use (outputs must be given)."""
        arrays, scalars, outs = self._split(args)
        ds, _ = self._marshal(arrays, scalars)
        os_ = [desc(o) for o in outs]
        need = C.c_size_t(0)
        ax = _axis_code(axis, max((a.ndim if isinstance(a, ChnArray) else a.dim()) for a in arrays if a is not None))
        _check(lib().chn_user_kernel_source(self._h, len(ds), _ptrs(ds), len(os_), _ptrs(os_), ax, int(keepdims), None, 0, C.byref(need)))
        buf = C.create_string_buffer(need.value)
        _check(lib().chn_user_kernel_source(self._h, len(ds), _ptrs(ds), len(os_), _ptrs(os_), ax, int(keepdims), buf, need.value, None))
        return buf.value.decode()


class ElementwiseKernel(_UserKernel):
    """``kernel = ElementwiseKernel('float32 x, float32 y, float32 z', 'float32 w', 'w = x * y + z',
    'my_mad'); w = kernel(x, y, z)`` -- the figure "Example of a user-defined kernel"."""

    def __init__(self, in_params, out_params, operation, name="kernel", preamble=""):
        h = C.c_void_p(None)
        _check(lib().chn_elementwise_kernel_create(in_params.encode(), out_params.encode(), operation.encode(),
                                                   name.encode(), preamble.encode(), C.byref(h)))
        super().__init__(h, in_params, out_params, name)

    def _outputs(self, arrays, outs):
        if outs:
            return outs
        shape = torch.broadcast_shapes(*[tuple(a.shape) for a in arrays if a is not None])
        dev = next(a.device for a in arrays if a is not None)
        return [torch.empty(shape, dtype=self._out_dtype(j, arrays), device=dev) for j in range(len(self.out_params))]

    def prepare(self, *args):
        arrays, scalars, outs = self._split(args)
        ds, _ = self._marshal(arrays, scalars)
        os_ = [desc(o) for o in self._outputs(arrays, outs)]
        _check(lib().chn_elementwise_kernel_prepare(self._h, len(ds), _ptrs(ds), len(os_), _ptrs(os_)))

    def __call__(self, *args, stream=None):
        arrays, scalars, outs = self._split(args)
        outs = self._outputs(arrays, outs)
        ds, sc = self._marshal(arrays, scalars)
        os_ = [desc(o) for o in outs]
        _check(lib().chn_elementwise_kernel_launch(self._h, len(ds), _ptrs(ds), len(os_), _ptrs(os_), sc,
                                                   _stream() if stream is None else stream))
        return outs[0] if len(outs) == 1 else tuple(outs)


class ReductionKernel(_UserKernel):
    """``ReductionKernel('T x', 'T y', 'x * x', 'a + b', 'y = sqrt(a)', '0', 'l2norm')(x, axis=1)``:
    fold map_expr of every element by reduce_expr from `identity`, then post_map_expr."""

    def __init__(self, in_params, out_params, map_expr, reduce_expr, post_map_expr, identity, name="reduce", preamble=""):
        h = C.c_void_p(None)
        _check(lib().chn_reduction_kernel_create(in_params.encode(), out_params.encode(), map_expr.encode(),
                                                 reduce_expr.encode(), post_map_expr.encode(), str(identity).encode(),
                                                 name.encode(), preamble.encode(), C.byref(h)))
        super().__init__(h, in_params, out_params, name)

    def _outputs(self, arrays, outs, axis, keepdims):
        if outs:
            return outs
        shape = list(torch.broadcast_shapes(*[tuple(a.shape) for a in arrays if a is not None]))
        axes = range(len(shape)) if axis is None else [a % len(shape) for a in (axis if isinstance(axis, (tuple, list)) else [axis])]
        oshape = [1 if d in axes else n for d, n in enumerate(shape)] if keepdims else [n for d, n in enumerate(shape) if d not in axes]
        dev = next(a.device for a in arrays if a is not None)
        return [torch.empty(oshape, dtype=self._out_dtype(j, arrays), device=dev) for j in range(len(self.out_params))]

    @staticmethod
    def _ndim(arrays):
        return max((a.ndim if isinstance(a, ChnArray) else a.dim()) for a in arrays if a is not None)

    def prepare(self, *args, axis=None, keepdims=False):
        arrays, scalars, outs = self._split(args)
        ds, _ = self._marshal(arrays, scalars)
        os_ = [desc(o) for o in self._outputs(arrays, outs, axis, keepdims)]
        _check(lib().chn_reduction_kernel_prepare(self._h, len(ds), _ptrs(ds), len(os_), _ptrs(os_),
                                                  _axis_code(axis, self._ndim(arrays)), int(keepdims)))

    def __call__(self, *args, axis=None, keepdims=False, ws=None, stream=None):
        arrays, scalars, outs = self._split(args)
        outs = self._outputs(arrays, outs, axis, keepdims)
        ds, sc = self._marshal(arrays, scalars)
        os_ = [desc(o) for o in outs]
        ax = _axis_code(axis, self._ndim(arrays))
        if ws is None:
            need = lib().chn_reduction_kernel_workspace_bytes(self._h, len(ds), _ptrs(ds), len(os_), _ptrs(os_), ax, int(keepdims))
            if need:
                ws = torch.empty(need, dtype=torch.uint8, device=outs[0].device)
        p, n = _ws(ws)
        _check(lib().chn_reduction_kernel_launch(self._h, len(ds), _ptrs(ds), len(os_), _ptrs(os_), sc, ax, int(keepdims),
                                                 p, n, _stream() if stream is None else stream))
        return outs[0] if len(outs) == 1 else tuple(outs)
