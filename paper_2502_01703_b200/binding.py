"""Thin Python binding of the C ABI in ``include/qless.h``.

Every function has the name of the C entry point it calls and does argument marshalling only:
torch supplies device memory and the current CUDA stream, the arithmetic runs in the library's
kernels. If ``libqless.so`` has not been built, or a call returns a non-OK status, an exception is
raised; there is no other code path.

``stream=`` runs a call on that stream instead of the current one. The caller orders the two (inputs
written on the current stream, results read there); memory that the binding allocates for the call
comes from that stream's pool, and the call's tensors are recorded as used on it.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqless.so")

QLESS_OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = 1, 2, 3, 4, 5
F32, BF16 = 0, 1
COSINE, DEQUANT = 0, 1

EXPORTS = [
    "qless_last_error", "qless_check", "qless_project_quantize_workspace", "qless_project_quantize",
    "qless_quantize", "qless_quantize_absmean", "qless_adam_gamma", "qless_philox_entries", "qless_score_workspace", "qless_score",
    "qless_score_16bit_workspace", "qless_score_16bit", "qless_inv_norms_16bit", "qless_score_dots_workspace", "qless_score_dots", "qless_select_topk_workspace", "qless_select_topk",
    "qless_project_quantize_host_workspace", "qless_project_quantize_host", "qless_profile_enable",
    "qless_profile_collect", "qless_kernel_launches", "qless_select_topk_static",
    "qless_set_projection_path", "qless_set_score_path", "qless_set_select_path", "qless_microbench",
    "qless_project_quantize_ex", "qless_project_quantize_host_ex", "qless_gaussian_entries", "qless_selftest_timeout",
    "qless_activation_quantize", "qless_activation_dequantize", "qless_lora_gradients_workspace", "qless_lora_gradients",
    "qless_lm_loss_workspace", "qless_lm_loss",
    "qless_layer_norm_backward_workspace", "qless_layer_norm", "qless_layer_norm_backward",
    "qless_attention_workspace", "qless_attention_backward_workspace", "qless_attention", "qless_attention_backward",
    "qless_gated_ffn_workspace", "qless_gated_ffn_backward_workspace", "qless_gated_ffn", "qless_gated_ffn_backward",
]
SILU, GELU = 0, 1
RADEMACHER, GAUSSIAN = 0, 1
SELECT_STATIC_MAX_N = 1 << 22


class AdamCfg(C.Structure):
    _fields_ = [("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float), ("step", C.c_int64)]


class ProjectionCfg(C.Structure):
    _fields_ = [("matrix", C.c_int32), ("reserved", C.c_int32 * 3)]


class QlessError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"qless status {status}: {message}")
        self.status = status


_lib = None


def lib():
    """The loaded shared library (loads it on first use; raises if it is missing)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} not found: build the CUDA library first (python -m paper_2502_01703_b200.build)")
        L = C.CDLL(LIB_PATH)
        vp, i64, i32, u64, sz = C.c_void_p, C.c_int64, C.c_int32, C.c_uint64, C.c_size_t
        L.qless_last_error.restype = C.c_char_p
        L.qless_last_error.argtypes = []
        L.qless_check.restype = C.c_int
        L.qless_check.argtypes = [vp]
        L.qless_project_quantize_workspace.restype = sz
        L.qless_project_quantize_workspace.argtypes = [i64, i64, i32, i32]
        L.qless_project_quantize.restype = C.c_int
        L.qless_project_quantize.argtypes = [vp, C.c_int, i64, i64, vp, vp, C.POINTER(AdamCfg), i64, i32, u64, i32,
                                             vp, vp, vp, vp, vp, sz, vp]
        L.qless_project_quantize_host_workspace.restype = sz
        L.qless_project_quantize_host_workspace.argtypes = [i64, i64, i32, i32, C.c_int]
        L.qless_project_quantize_host.restype = C.c_int
        L.qless_project_quantize_host.argtypes = [vp, C.c_int, i64, i64, vp, vp, C.POINTER(AdamCfg), i64, i32, u64, i32,
                                                  vp, vp, vp, vp, sz, vp]
        L.qless_profile_enable.restype = C.c_int
        L.qless_profile_enable.argtypes = [i32]
        L.qless_kernel_launches.restype = C.c_uint64
        L.qless_kernel_launches.argtypes = []
        L.qless_profile_collect.restype = C.c_int
        L.qless_profile_collect.argtypes = [C.c_char_p, sz]
        L.qless_quantize.restype = C.c_int
        L.qless_quantize.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, vp]
        L.qless_quantize_absmean.restype = C.c_int
        L.qless_quantize_absmean.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, vp]
        L.qless_adam_gamma.restype = C.c_int
        L.qless_adam_gamma.argtypes = [vp, C.c_int, i64, i64, vp, vp, C.POINTER(AdamCfg), i64, vp, vp]
        L.qless_philox_entries.restype = C.c_int
        L.qless_philox_entries.argtypes = [u64, i64, i64, i64, i64, vp, vp]
        L.qless_score_workspace.restype = sz
        L.qless_score_workspace.argtypes = [i64, i32, i32, i32, i32, i32]
        L.qless_score.restype = C.c_int
        L.qless_score.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, C.POINTER(C.c_float), C.POINTER(i32),
                                  i64, i32, i32, i32, i32, i32, C.c_int, vp, vp, vp, sz, vp]
        L.qless_score_16bit_workspace.restype = sz
        L.qless_score_16bit_workspace.argtypes = [i64, i32, i32, i32]
        L.qless_score_16bit.restype = C.c_int
        L.qless_score_16bit.argtypes = [vp, i64, vp, i64, vp, vp, C.POINTER(C.c_float), C.POINTER(i32), i64, i32, i32, i32,
                                        i32, vp, vp, vp, sz, vp]
        L.qless_inv_norms_16bit.restype = C.c_int
        L.qless_inv_norms_16bit.argtypes = [vp, i64, i64, i32, i32, vp, vp]
        L.qless_score_dots_workspace.restype = sz
        L.qless_score_dots_workspace.argtypes = [i64, i32, i32, i32]
        L.qless_score_dots.restype = C.c_int
        L.qless_score_dots.argtypes = [vp, vp, i64, i64, i32, i32, i32, vp, vp, sz, vp]
        L.qless_select_topk_workspace.restype = sz
        L.qless_select_topk_workspace.argtypes = [i64]
        L.qless_select_topk.restype = C.c_int
        L.qless_select_topk.argtypes = [vp, i64, C.c_double, vp, C.POINTER(i64), vp, sz, vp]
        L.qless_microbench.restype = C.c_int
        L.qless_microbench.argtypes = [i32, i32, C.POINTER(C.c_float), C.POINTER(C.c_double), vp, sz, vp]
        L.qless_set_score_path.restype = C.c_int
        L.qless_set_score_path.argtypes = [i32]
        L.qless_set_select_path.restype = C.c_int
        L.qless_set_select_path.argtypes = [i32]
        L.qless_set_projection_path.restype = C.c_int
        L.qless_set_projection_path.argtypes = [i32]
        L.qless_project_quantize_ex.restype = C.c_int
        L.qless_project_quantize_ex.argtypes = [vp, C.c_int, i64, i64, vp, vp, C.POINTER(AdamCfg), i64, i32, u64,
                                                C.POINTER(ProjectionCfg), i32, vp, vp, vp, vp, vp, sz, vp]
        L.qless_project_quantize_host_ex.restype = C.c_int
        L.qless_project_quantize_host_ex.argtypes = [vp, C.c_int, i64, i64, vp, vp, C.POINTER(AdamCfg), i64, i32, u64,
                                                     C.POINTER(ProjectionCfg), i32, vp, vp, vp, vp, sz, vp]
        L.qless_selftest_timeout.restype = C.c_int
        L.qless_selftest_timeout.argtypes = [i32, vp]
        L.qless_gaussian_entries.restype = C.c_int
        L.qless_gaussian_entries.argtypes = [C.c_uint64, i64, i64, i64, i64, vp, vp]
        L.qless_select_topk_static.restype = C.c_int
        L.qless_select_topk_static.argtypes = [vp, i64, C.c_double, vp, C.POINTER(i64), vp]
        L.qless_activation_quantize.restype = C.c_int
        L.qless_activation_quantize.argtypes = [vp, C.c_int, i64, i32, i64, i32, vp, i64, vp, i64, vp]
        L.qless_activation_dequantize.restype = C.c_int
        L.qless_activation_dequantize.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, C.c_int, i64, vp]
        L.qless_lora_gradients_workspace.restype = sz
        L.qless_lora_gradients_workspace.argtypes = [i64, i64, i32, i32, i32, C.c_int]
        L.qless_lora_gradients.restype = C.c_int
        L.qless_lora_gradients.argtypes = [vp, i64, vp, i64, i32, vp, i64, vp, vp, vp, i64, i64, i32, i32, i32, C.c_float, vp, C.c_int,
                                           i64, vp, sz, vp]
        L.qless_lm_loss_workspace.restype = sz
        L.qless_lm_loss_workspace.argtypes = [i64, i32, i32, i32, i32]
        L.qless_lm_loss.restype = C.c_int
        L.qless_lm_loss.argtypes = [vp, i64, vp, i64, vp, vp, i64, i32, i32, vp, vp, i64, vp, i64, vp, sz, vp]
        fp = C.c_float
        for name, result, args in (
                ("qless_layer_norm_backward_workspace", sz, [i64, i32, i32]),
                ("qless_layer_norm", C.c_int, [vp, C.c_int, i64, i32, i64, vp, vp, C.c_int, fp, i32, vp, i64, vp, vp, vp]),
                ("qless_layer_norm_backward", C.c_int, [vp, i64, vp, C.c_int, i64, i32, i64, vp, C.c_int, i32, vp, vp, vp, i64, vp, vp, vp, sz, vp]),
                ("qless_attention_workspace", sz, [i64, i64, i32, i32]),
                ("qless_attention_backward_workspace", sz, [i64, i64, i32, i32]),
                ("qless_attention", C.c_int, [vp, i64] * 3 + [vp, i64, i64, i32, i32, i32, fp, vp, i64, vp, vp, sz, vp]),
                ("qless_attention_backward", C.c_int, [vp, i64] * 5 + [vp, vp, i64, i64, i32, i32, i32, fp] + [vp, i64] * 3 + [vp, sz, vp]),
                ("qless_gated_ffn_workspace", sz, [i64, i32, i32]),
                ("qless_gated_ffn_backward_workspace", sz, [i64, i32, i32, i32]),
                ("qless_gated_ffn", C.c_int, [vp, i64] * 4 + [i64, i32, i32, C.c_int] + [vp, i64] * 4 + [vp, sz, vp]),
                ("qless_gated_ffn_backward", C.c_int, [vp, i64] * 7 + [i64, i32, i32, C.c_int] + [vp, i64] * 6 + [vp, sz, vp])):
            fn = getattr(L, name)
            fn.restype, fn.argtypes = result, args
        _lib = L
    return _lib


def _check(status):
    if status != QLESS_OK:
        raise QlessError(status, lib().qless_last_error().decode())


def _ptr(t):
    return t.data_ptr() if t is not None else None


# The raw handle of a device's current stream without building a Stream object for every call. Not part of torch's public interface:
# a build of torch that lacks it takes the public way.
_raw_current = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None, device=None):
    """The stream's raw handle; None: that of the current stream (device: the current one, where the caller has asked already)."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_current is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_current(torch.cuda.current_device() if device is None else device)


def _dtype_code(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("gradients must be float32 or bfloat16")


def _adam(adam):
    if adam is None:
        return None
    return C.byref(AdamCfg(adam.get("beta1", 0.9), adam.get("beta2", 0.999), adam.get("eps", 1e-8),
                           int(adam.get("step", 0))))


def _projection(matrix):
    return C.byref(ProjectionCfg(int(matrix), (C.c_int32 * 3)(0, 0, 0)))


def _elsewhere(stream):
    """True where a call is asked to run on another stream than the current one."""
    return stream is not None and stream.cuda_stream != _stream()


def _new(shape, dtype, device, stream):
    """A new contiguous output of a call on `stream`. Where that is not the current stream, the memory comes from that stream's pool: a
    block of the current stream's pool might still be in use there when the kernels begin. The current stream, on which the
    caller is likely to read the result, is recorded as a user of it."""
    if not _elsewhere(stream):
        return torch.empty(shape, dtype=dtype, device=device)
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if t.is_cuda:
        t.record_stream(here)
    return t


def _used(stream, *tensors):
    """Records a call's tensors (None: absent) as used on `stream`, so that one that is dropped as soon as the call returns is not given
    out again on the current stream while the kernels still run."""
    if _elsewhere(stream):
        for t in tensors:
            if t is not None and t.is_cuda:
                t.record_stream(stream)


def _workspace(nbytes, device, workspace, stream):
    if workspace is not None:
        return workspace
    nbytes = max(int(nbytes), 256)
    if not _elsewhere(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):        # goes back to that stream's pool when the call returns: reused behind the kernels only
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _workspace_if(nbytes, device, workspace, stream):
    """(pointer, size, tensor) of a call's workspace: none where it needs none."""
    if workspace is None:
        if nbytes == 0:
            return None, 0, None
        workspace = _workspace(nbytes, device, None, stream)
    return workspace.data_ptr(), workspace.numel(), workspace


def qless_last_error():
    return lib().qless_last_error().decode()


def qless_check(stream=None):
    _check(lib().qless_check(_stream(stream)))


def qless_project_quantize_workspace(n, P, d, bits):
    return int(lib().qless_project_quantize_workspace(n, P, d, bits))


def qless_project_quantize(grads, d, seed, bits, adam_m=None, adam_v=None, adam=None, want_sumsq=True,
                           want_proj=False, out=None, workspace=None, stream=None, matrix=None):
    """grads [n, P] f32/bf16 (row stride allowed) -> dict(codes uint8 [n, d*bits/8], scales f32 [n],
    sumsq i32 [n] | None, proj f32 [n, d] | None). `out` may pass preallocated tensors by those names.
    matrix = None calls qless_project_quantize; RADEMACHER / GAUSSIAN call qless_project_quantize_ex with that
    matrix in its projection config."""
    n, P = grads.shape
    dev = grads.device
    out = out or {}
    codes = out.get("codes", None)
    if codes is None:
        codes = _new((n, d * bits // 8), torch.uint8, dev, stream)
    scales = out.get("scales", None)
    if scales is None:
        scales = _new(n, torch.float32, dev, stream)
    sumsq = out.get("sumsq", _new(n, torch.int32, dev, stream) if want_sumsq else None)
    proj = out.get("proj", _new((n, d), torch.float32, dev, stream) if want_proj else None)
    ws = _workspace(qless_project_quantize_workspace(n, P, d, bits), dev, workspace, stream)
    _used(stream, grads, adam_m, adam_v, workspace, *out.values())
    if matrix is None:
        _check(lib().qless_project_quantize(_ptr(grads), _dtype_code(grads), n, grads.stride(0) if n > 0 else P,
                                            _ptr(adam_m), _ptr(adam_v), _adam(adam), P, d, seed, bits,
                                            _ptr(codes), _ptr(scales), _ptr(sumsq), _ptr(proj),
                                            _ptr(ws), ws.numel(), _stream(stream)))
    else:
        _check(lib().qless_project_quantize_ex(_ptr(grads), _dtype_code(grads), n, grads.stride(0) if n > 0 else P,
                                               _ptr(adam_m), _ptr(adam_v), _adam(adam), P, d, seed, _projection(matrix),
                                               bits, _ptr(codes), _ptr(scales), _ptr(sumsq), _ptr(proj),
                                               _ptr(ws), ws.numel(), _stream(stream)))
    return dict(codes=codes, scales=scales, sumsq=sumsq, proj=proj)


def qless_project_quantize_host_workspace(n, P, d, bits, dtype_code):
    return int(lib().qless_project_quantize_host_workspace(n, P, d, bits, dtype_code))


def qless_project_quantize_host(grads_host, d, seed, bits, adam_m=None, adam_v=None, adam=None, out=None,
                                workspace=None, device="cuda", stream=None, matrix=None):
    """grads_host: CPU tensor [n, P] (pinned for asynchronous copies); adam_m / adam_v: device tensors.
    Returns dict(codes, scales, sumsq) of CPU tensors (pinned), valid once the stream has drained."""
    n, P = grads_host.shape
    out = out or {}
    codes = out.get("codes")
    if codes is None:
        codes = torch.empty((n, d * bits // 8), dtype=torch.uint8).pin_memory()
    scales = out.get("scales")
    if scales is None:
        scales = torch.empty(n, dtype=torch.float32).pin_memory()
    sumsq = out.get("sumsq")
    if sumsq is None:
        sumsq = torch.empty(n, dtype=torch.int32).pin_memory()
    code = _dtype_code(grads_host)
    ws = _workspace(qless_project_quantize_host_workspace(n, P, d, bits, code), device, workspace, stream)
    _used(stream, adam_m, adam_v, workspace)
    if matrix is None:
        _check(lib().qless_project_quantize_host(_ptr(grads_host), code, n, grads_host.stride(0) if n > 0 else P,
                                                 _ptr(adam_m), _ptr(adam_v), _adam(adam), P, d, seed, bits,
                                                 _ptr(codes), _ptr(scales), _ptr(sumsq), _ptr(ws), ws.numel(),
                                                 _stream(stream)))
    else:
        _check(lib().qless_project_quantize_host_ex(_ptr(grads_host), code, n, grads_host.stride(0) if n > 0 else P,
                                                    _ptr(adam_m), _ptr(adam_v), _adam(adam), P, d, seed,
                                                    _projection(matrix), bits, _ptr(codes), _ptr(scales), _ptr(sumsq),
                                                    _ptr(ws), ws.numel(), _stream(stream)))
    return dict(codes=codes, scales=scales, sumsq=sumsq)


def qless_profile_enable(on=True):
    _check(lib().qless_profile_enable(1 if on else 0))


def qless_kernel_launches():
    return int(lib().qless_kernel_launches())


def qless_profile_collect():
    """{kernel name: (total milliseconds, launches)} since the last collect."""
    buf = C.create_string_buffer(4096)
    _check(lib().qless_profile_collect(buf, 4096))
    out = {}
    for item in buf.value.decode().split(";"):
        if item:
            name, rest = item.split("=")
            ms, cnt = rest.split("*")
            out[name] = (float(ms), int(cnt))
    return out


def qless_quantize(x, bits, normalize=True, want_sumsq=True, stream=None):
    n, d = x.shape
    dev = x.device
    codes = _new((n, d * bits // 8), torch.uint8, dev, stream)
    scales = _new(n, torch.float32, dev, stream)
    sumsq = _new(n, torch.int32, dev, stream) if want_sumsq else None
    _used(stream, x)
    _check(lib().qless_quantize(_ptr(x), n, d, 1 if normalize else 0, bits, _ptr(codes), _ptr(scales),
                                _ptr(sumsq), _stream(stream)))
    return codes, scales, sumsq


def qless_quantize_absmean(x, bits, normalize=True, want_sumsq=True, stream=None):
    """As qless_quantize, with the scale taken from the mean absolute value of the row."""
    n, d = x.shape
    dev = x.device
    codes = _new((n, d * bits // 8), torch.uint8, dev, stream)
    scales = _new(n, torch.float32, dev, stream)
    sumsq = _new(n, torch.int32, dev, stream) if want_sumsq else None
    _used(stream, x)
    _check(lib().qless_quantize_absmean(_ptr(x), n, d, 1 if normalize else 0, bits, _ptr(codes), _ptr(scales),
                                        _ptr(sumsq), _stream(stream)))
    return codes, scales, sumsq


def qless_adam_gamma(grads, adam_m=None, adam_v=None, adam=None, stream=None):
    n, P = grads.shape
    out = _new((n, P), torch.bfloat16, grads.device, stream)
    _used(stream, grads, adam_m, adam_v)
    _check(lib().qless_adam_gamma(_ptr(grads), _dtype_code(grads), n, grads.stride(0) if n > 0 else P,
                                  _ptr(adam_m), _ptr(adam_v), _adam(adam), P, _ptr(out), _stream(stream)))
    return out


def qless_philox_entries(seed, r0, nr, j0, nj, device="cuda", stream=None):
    out = _new((nr, nj), torch.int8, device, stream)
    _check(lib().qless_philox_entries(seed, r0, nr, j0, nj, _ptr(out), _stream(stream)))
    return out


def qless_gaussian_entries(seed, r0, nr, j0, nj, device="cuda", stream=None):
    out = _new((nr, nj), torch.float32, device, stream)
    _check(lib().qless_gaussian_entries(seed, r0, nr, j0, nj, _ptr(out), _stream(stream)))
    return out


def qless_score_workspace(N, V, Cn, T, d, bits):
    return int(lib().qless_score_workspace(N, V, Cn, T, d, bits))


def qless_score(train_codes, val_codes, train_scales, val_scales, lr_weights, task_offsets, d, bits,
                train_sumsq=None, val_sumsq=None, mode=COSINE, want_per_task=False, scores=None,
                workspace=None, stream=None):
    """train_codes uint8 [C, N, d*bits/8], val_codes uint8 [C, V, d*bits/8] (checkpoint stride taken from
    the tensors), scales f32 [C, N] / [C, V]; lr_weights / task_offsets: host sequences."""
    Cn, N, rb = train_codes.shape
    V = val_codes.shape[1]
    dev = train_codes.device
    T = len(task_offsets) - 1
    eta = (C.c_float * Cn)(*[float(x) for x in lr_weights])
    off = (C.c_int32 * (T + 1))(*[int(x) for x in task_offsets])
    if scores is None:
        scores = _new(N, torch.float32, dev, stream)
    per_task = _new((N, T), torch.float32, dev, stream) if want_per_task else None
    ws = _workspace(qless_score_workspace(N, V, Cn, T, d, bits), dev, workspace, stream)
    _used(stream, train_codes, val_codes, train_scales, val_scales, train_sumsq, val_sumsq, scores, workspace)
    _check(lib().qless_score(_ptr(train_codes), train_codes.stride(0) if Cn > 0 else 0,
                             _ptr(val_codes), val_codes.stride(0),
                             _ptr(train_scales), _ptr(val_scales), _ptr(train_sumsq), _ptr(val_sumsq),
                             eta, off, N, V, Cn, T, d, bits, mode, _ptr(scores), _ptr(per_task),
                             _ptr(ws), ws.numel(), _stream(stream)))
    return (scores, per_task) if want_per_task else scores


def qless_score_16bit_workspace(N, V, Cn, T):
    return int(lib().qless_score_16bit_workspace(N, V, Cn, T))


def qless_inv_norms_16bit(rows, stream=None):
    """rows bf16 [C, n, d] -> 1 / ||row|| as f32 [C, n] (0 for a zero row)."""
    Cn, n, d = rows.shape
    out = _new((Cn, n), torch.float32, rows.device, stream)
    _used(stream, rows)
    _check(lib().qless_inv_norms_16bit(_ptr(rows), rows.stride(0) * 2, n, Cn, d, _ptr(out), _stream(stream)))
    return out


def qless_score_16bit(train_rows, val_rows, lr_weights, task_offsets, want_per_task=False, scores=None,
                      workspace=None, stream=None, train_inv_norms=None, val_inv_norms=None):
    """The 16-bit baseline: train_rows bf16 [C, N, d], val_rows bf16 [C, V, d] (checkpoint stride taken from the
    tensors); lr_weights / task_offsets: host sequences."""
    assert train_rows.dtype == torch.bfloat16 and val_rows.dtype == torch.bfloat16
    Cn, N, d = train_rows.shape
    V = val_rows.shape[1]
    dev = train_rows.device
    T = len(task_offsets) - 1
    eta = (C.c_float * Cn)(*[float(x) for x in lr_weights])
    off = (C.c_int32 * (T + 1))(*[int(x) for x in task_offsets])
    if scores is None:
        scores = _new(N, torch.float32, dev, stream)
    per_task = _new((N, T), torch.float32, dev, stream) if want_per_task else None
    ws = _workspace(qless_score_16bit_workspace(N, V, Cn, T), dev, workspace, stream)
    _used(stream, train_rows, val_rows, train_inv_norms, val_inv_norms, scores, workspace)
    _check(lib().qless_score_16bit(_ptr(train_rows), train_rows.stride(0) * 2 if Cn > 0 else 0, _ptr(val_rows),
                                   val_rows.stride(0) * 2, _ptr(train_inv_norms), _ptr(val_inv_norms), eta, off, N, V, Cn, T,
                                   d, _ptr(scores), _ptr(per_task),
                                   _ptr(ws), ws.numel(), _stream(stream)))
    return (scores, per_task) if want_per_task else scores


def qless_score_dots_workspace(nt, V, d, bits):
    return int(lib().qless_score_dots_workspace(nt, V, d, bits))


def qless_score_dots(train_codes, val_codes, d, bits, t0=0, nt=None, workspace=None, stream=None):
    """One checkpoint: train_codes uint8 [N, rb], val_codes uint8 [V, rb] -> int32 [nt, V]."""
    if nt is None:
        nt = train_codes.shape[0] - t0
    V = val_codes.shape[0]
    dev = train_codes.device
    dots = _new((nt, V), torch.int32, dev, stream)
    ws = _workspace(qless_score_dots_workspace(nt, V, d, bits), dev, workspace, stream)
    _used(stream, train_codes, val_codes, workspace)
    _check(lib().qless_score_dots(_ptr(train_codes), _ptr(val_codes), t0, nt, V, d, bits, _ptr(dots),
                                  _ptr(ws), ws.numel(), _stream(stream)))
    return dots


def qless_select_topk_workspace(N):
    return int(lib().qless_select_topk_workspace(N))


def qless_select_topk(scores, frac, indices=None, workspace=None, stream=None):
    """scores f32 [N] -> int64 [k] ascending indices of the top floor(frac*N) scores."""
    N = scores.numel()
    dev = scores.device
    if indices is None:
        indices = _new(max(N, 1), torch.int64, dev, stream)
    ws = _workspace(qless_select_topk_workspace(N), dev, workspace, stream)
    _used(stream, scores, indices, workspace)
    k = C.c_int64(0)
    _check(lib().qless_select_topk(_ptr(scores), N, float(frac), _ptr(indices), C.byref(k), _ptr(ws),
                                   ws.numel(), _stream(stream)))
    return indices[:k.value]


def qless_select_topk_static(scores, frac, indices, stream=None):
    """Allocation-free variant of qless_select_topk for N <= SELECT_STATIC_MAX_N: the scratch is a fixed
    array inside the library, so the caller passes only the input and a preallocated int64 `indices`
    tensor with room for k entries. Returns a view of the first k entries; nothing is allocated here
    either. Calls that overlap on the GPU share that array and must be serialised by the caller."""
    _used(stream, scores, indices)
    k = C.c_int64(0)
    _check(lib().qless_select_topk_static(_ptr(scores), scores.numel(), float(frac), _ptr(indices), C.byref(k),
                                          _stream(stream)))
    return indices[:k.value]


def _row_stride(t):
    """Elements between rows of a 2-D tensor whose rows are contiguous."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("a 2-D tensor with contiguous rows is required")
    # what a single row's stride says means nothing (torch calls such a tensor contiguous whatever it is): the next multiple of 16 will do
    return stride[0] if shape[0] > 1 else -(-shape[1] // 16) * 16


def _on_gpu(stream, *tensors):
    """The GPU that a call runs on. Refuses tensors (None: absent) that its kernels cannot read: in host memory, or on another GPU than its
    stream. Outputs that the binding has just made beside an input need no look."""
    at = tensors[0].get_device()
    for t in tensors:
        if t is not None and (at < 0 or t.get_device() != at):
            raise ValueError("all tensors must be on one GPU")
    if at != (torch.cuda.current_device() if stream is None else stream.device_index):
        raise ValueError("the tensors must be on the GPU of the stream")
    return at


def _empty(rows, cols, dtype, device, stream):
    """A new contiguous [rows, cols] output (the strided form of torch.empty takes two thirds of its time)."""
    if stream is None:
        return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)
    return _new((rows, cols), dtype, device, stream)


def _line(n, dtype, device, stream):
    if stream is None:
        return torch.empty_strided((n,), (1,), dtype=dtype, device=device)
    return _new(n, dtype, device, stream)


def _dtype_of(dtype):
    if dtype == torch.float32:
        return F32
    if dtype == torch.bfloat16:
        return BF16
    raise TypeError("float32 or bfloat16 is required")


def qless_activation_quantize(x, group=32, codes=None, scales=None, stream=None):
    """x f32/bf16 [tokens, width] (row stride allowed) -> (codes int8 [tokens, width], scales uint8
    [tokens, ceil(width / group)]): the 8-bit checkpoint of a layer's input, one power-of-two step per group of channels."""
    T, width = x.shape
    groups = -(-width // max(int(group), 1))
    at = _on_gpu(stream, x, codes, scales) if codes is not None or scales is not None else _on_gpu(stream, x)
    if codes is None:
        codes = _empty(T, width, torch.int8, x.device, stream)
    elif codes.shape != (T, width) or codes.dtype != torch.int8:
        raise ValueError("codes must be int8 [tokens, width]")
    if scales is None:
        scales = _empty(T, groups, torch.uint8, x.device, stream)
    elif scales.shape != (T, groups) or scales.dtype != torch.uint8:
        raise ValueError("scales must be uint8 [tokens, ceil(width / group)]")
    if stream is not None:
        _used(stream, x, codes, scales)
    _check(lib().qless_activation_quantize(x.data_ptr(), _dtype_code(x), T, width, _row_stride(x), group, codes.data_ptr(), _row_stride(codes),
                                           scales.data_ptr(), _row_stride(scales), _stream(stream, at)))
    return codes, scales


def qless_activation_dequantize(codes, scales, group=32, dtype=torch.bfloat16, out=None, stream=None):
    """The values that a checkpoint's codes stand for, [tokens, width] of `dtype` (exact in both types)."""
    T, width = codes.shape
    if codes.dtype != torch.int8 or scales.dtype != torch.uint8 or scales.shape != (T, -(-width // max(int(group), 1))):
        raise ValueError("codes must be int8 [tokens, width] and scales uint8 [tokens, ceil(width / group)]")
    at = _on_gpu(stream, codes, scales, out)
    if out is None:
        out = _empty(T, width, dtype, codes.device, stream)
    elif out.shape != (T, width):
        raise ValueError("out must be [tokens, width]")
    if stream is not None:
        _used(stream, codes, scales, out)
    _check(lib().qless_activation_dequantize(_ptr(codes), _row_stride(codes), _ptr(scales), _row_stride(scales), T, width, group,
                                             _ptr(out), _dtype_code(out), _row_stride(out), _stream(stream, at)))
    return out


def qless_lora_gradients_workspace(tokens, n, width_in, width_out, rank, dtype=torch.bfloat16):
    return int(lib().qless_lora_gradients_workspace(tokens, n, width_in, width_out, rank, _dtype_of(dtype)))


def qless_lora_gradients(codes, scales, grad_out, lora_a, lora_b, offsets, scaling=1.0, group=32, grads=None, dtype=torch.bfloat16,
                         workspace=None, stream=None):
    """Per-example LoRA gradients of one layer from its 8-bit input checkpoint: codes int8 [tokens, in], scales uint8,
    grad_out bf16 [tokens, out], lora_a bf16 [rank, in], lora_b bf16 [out, rank]; offsets: int64 CPU tensor (or sequence)
    [n + 1] of the examples' first tokens. Returns grads [n, rank * (in + out)], rows [dA | dB]; `grads` may be a column
    slice of a wider [n, P] matrix."""
    off = offsets if torch.is_tensor(offsets) else torch.tensor(list(offsets), dtype=torch.int64)
    if off.device.type != "cpu" or off.dtype != torch.int64 or not off.is_contiguous():
        raise TypeError("offsets must be a contiguous int64 tensor in host memory")
    if grad_out.dtype != torch.bfloat16 or lora_a.dtype != torch.bfloat16 or lora_b.dtype != torch.bfloat16:
        raise TypeError("grad_out, lora_a and lora_b must be bfloat16")
    if codes.dtype != torch.int8 or scales.dtype != torch.uint8:
        raise TypeError("codes must be int8 and scales uint8")
    T, wi = codes.shape
    rank, wo = lora_a.shape[0], lora_b.shape[0]
    n = off.numel() - 1
    if grad_out.shape != (T, wo) or lora_a.shape[1] != wi or lora_b.shape[1] != rank or scales.shape != (T, -(-wi // max(int(group), 1))):
        raise ValueError("shapes of codes, scales, grad_out, lora_a and lora_b do not fit together")
    if not lora_a.is_contiguous() or not lora_b.is_contiguous():
        raise ValueError("lora_a and lora_b must be contiguous")
    if grads is None:
        grads = _empty(n, rank * (wi + wo), dtype, codes.device, stream)
    elif grads.shape != (n, rank * (wi + wo)):
        raise ValueError("grads must be [n, rank * (in + out)]")
    at = _on_gpu(stream, codes, scales, grad_out, lora_a, lora_b, grads, workspace)
    ws = _workspace(qless_lora_gradients_workspace(T, n, wi, wo, rank, grads.dtype), codes.device, workspace, stream)
    if stream is not None:
        _used(stream, codes, scales, grad_out, lora_a, lora_b, grads, workspace)
    _check(lib().qless_lora_gradients(_ptr(codes), _row_stride(codes), _ptr(scales), _row_stride(scales), group, _ptr(grad_out),
                                      _row_stride(grad_out), _ptr(lora_a), _ptr(lora_b), _ptr(off), T, n, wi, wo, rank, scaling,
                                      _ptr(grads), _dtype_code(grads), _row_stride(grads), _ptr(ws), ws.numel(), _stream(stream, at)))
    return grads


def qless_lm_loss_workspace(tokens, width, vocab, want_hidden=True, want_weight=False):
    return int(lib().qless_lm_loss_workspace(tokens, width, vocab, 1 if want_hidden else 0, 1 if want_weight else 0))


def qless_lm_loss(hidden, weight, labels, token_weight=None, want_hidden=True, want_weight=False, out=None, workspace=None, stream=None):
    """Softmax cross entropy over a large vocabulary with its gradient: hidden bf16 [tokens, width], weight bf16 [vocab, width],
    labels int64 [tokens] (outside [0, vocab): no loss), token_weight f32 [tokens] or None. Returns dict(loss f32 [tokens],
    grad_hidden bf16 [tokens, width] | None, grad_weight bf16 [vocab, width] | None), the gradients being those of
    sum(token_weight * loss). `out` may pass preallocated tensors by those names."""
    if hidden.dtype != torch.bfloat16 or weight.dtype != torch.bfloat16:
        raise TypeError("hidden and weight must be bfloat16")
    if labels.dtype != torch.int64 or not labels.is_contiguous():
        raise TypeError("labels must be a contiguous int64 tensor")
    T, width = hidden.shape
    vocab = weight.shape[0]
    if weight.shape[1] != width or labels.shape != (T,):
        raise ValueError("shapes of hidden, weight and labels do not fit together")
    if token_weight is not None and (token_weight.dtype != torch.float32 or token_weight.shape != (T,) or not token_weight.is_contiguous()):
        raise ValueError("token_weight must be a contiguous float32 tensor [tokens]")
    dev = hidden.device
    out = out or {}
    loss = out.get("loss")
    if loss is None:
        loss = _new(T, torch.float32, dev, stream)
    gh = out.get("grad_hidden")
    if gh is None and want_hidden:
        gh = _empty(T, width, torch.bfloat16, dev, stream)
    gw = out.get("grad_weight")
    if gw is None and want_weight:
        gw = _empty(vocab, width, torch.bfloat16, dev, stream)
    for t, shape in ((loss, (T,)), (gh, (T, width)), (gw, (vocab, width))):
        if t is not None and (t.shape != shape or t.dtype != (torch.float32 if t is loss else torch.bfloat16)):
            raise ValueError("an output has the wrong shape or type")
    if not loss.is_contiguous():
        raise ValueError("loss must be contiguous")
    at = _on_gpu(stream, hidden, weight, labels, token_weight, loss, gh, gw, workspace)
    ws = _workspace(qless_lm_loss_workspace(T, width, vocab, gh is not None, gw is not None), dev, workspace, stream)
    if stream is not None:
        _used(stream, hidden, weight, labels, token_weight, loss, gh, gw, workspace)
    _check(lib().qless_lm_loss(_ptr(hidden), _row_stride(hidden), _ptr(weight), _row_stride(weight), _ptr(labels), _ptr(token_weight),
                               T, width, vocab, _ptr(loss), _ptr(gh), _row_stride(gh) if gh is not None else 0,
                               _ptr(gw), _row_stride(gw) if gw is not None else 0, _ptr(ws), ws.numel(), _stream(stream, at)))
    return dict(loss=loss, grad_hidden=gh, grad_weight=gw)


def _param(p, width, name):
    if p is not None and (p.shape != (width,) or not p.is_contiguous()):
        raise ValueError(f"{name} must be contiguous, [width]")
    return p


def qless_layer_norm(x, weight, bias=None, eps=1e-5, center=True, out=None, stream=None):
    """Layer normalisation of the rows of x f32/bf16 [tokens, width] (row stride allowed); weight, bias [width] f32 or bf16; center=False: by
    the root mean square. Returns dict(out [tokens, width] of x's type, mean f32 [tokens] | None without centring, rstd f32 [tokens])."""
    T, width = x.shape
    _param(weight, width, "weight")
    _param(bias, width, "bias")
    if bias is not None and bias.dtype != weight.dtype:
        raise TypeError("weight and bias must have one type")
    at = _on_gpu(stream, x, weight, bias, out)
    if out is None:
        out = _empty(T, width, x.dtype, x.device, stream)
    elif out.shape != (T, width) or out.dtype != x.dtype:
        raise ValueError("out must be [tokens, width] of x's type")
    mean = _line(T, torch.float32, x.device, stream) if center else None
    rstd = _line(T, torch.float32, x.device, stream)
    if stream is not None:
        _used(stream, x, weight, bias, out)
    _check(lib().qless_layer_norm(x.data_ptr(), _dtype_code(x), T, width, _row_stride(x), weight.data_ptr(), _ptr(bias), _dtype_code(weight), eps,
                                  1 if center else 0, out.data_ptr(), _row_stride(out), _ptr(mean), rstd.data_ptr(), _stream(stream, at)))
    return dict(out=out, mean=mean, rstd=rstd)


def qless_layer_norm_backward_workspace(tokens, width, want_params=True):
    return int(lib().qless_layer_norm_backward_workspace(tokens, width, 1 if want_params else 0))


def qless_layer_norm_backward(grad_out, x, weight, mean, rstd, want_weight=False, want_bias=False, grad_x=None, workspace=None, stream=None):
    """Gradients of qless_layer_norm from the mean (None: without centring) and rstd that it returned. Returns dict(grad_x [tokens, width] of
    x's type, grad_weight | None, grad_bias | None: [width] of weight's type)."""
    T, width = x.shape
    _param(weight, width, "weight")
    if grad_out.shape != (T, width) or grad_out.dtype != x.dtype:
        raise ValueError("grad_out must be [tokens, width] of x's type")
    for s in (mean, rstd):
        if s is not None and (s.shape != (T,) or s.dtype != torch.float32 or not s.is_contiguous()):
            raise ValueError("mean and rstd must be contiguous float32, [tokens]")
    at = _on_gpu(stream, x, grad_out, weight, mean, rstd, grad_x, workspace)
    if grad_x is None:
        grad_x = _empty(T, width, x.dtype, x.device, stream)
    elif grad_x.shape != (T, width) or grad_x.dtype != x.dtype:
        raise ValueError("grad_x must be [tokens, width] of x's type")
    gw = _line(width, weight.dtype, x.device, stream) if want_weight else None
    gb = _line(width, weight.dtype, x.device, stream) if want_bias else None
    ws, ws_bytes, _hold = _workspace_if(lib().qless_layer_norm_backward_workspace(T, width, 1) if want_weight or want_bias else 0, x.device, workspace, stream)
    if stream is not None:
        _used(stream, x, grad_out, weight, mean, rstd, grad_x, workspace)
    _check(lib().qless_layer_norm_backward(grad_out.data_ptr(), _row_stride(grad_out), x.data_ptr(), _dtype_code(x), T, width, _row_stride(x),
                                           weight.data_ptr(), _dtype_code(weight), 0 if mean is None else 1, _ptr(mean), rstd.data_ptr(),
                                           grad_x.data_ptr(), _row_stride(grad_x), _ptr(gw), _ptr(gb), ws, ws_bytes,
                                           _stream(stream, at)))
    return dict(grad_x=grad_x, grad_weight=gw, grad_bias=gb)


def _host_offsets(offsets):
    off = offsets if torch.is_tensor(offsets) else torch.tensor(list(offsets), dtype=torch.int64)
    if off.device.type != "cpu" or off.dtype != torch.int64 or not off.is_contiguous() or off.dim() != 1 or off.numel() < 1:
        raise TypeError("offsets must be a contiguous int64 tensor in host memory, [n + 1]")
    return off


def _token_stride(t, name):
    """Elements between tokens of a bf16 [tokens, heads, head_dim] tensor whose heads lie side by side."""
    shape, stride = t.shape, t.stride()
    if t.dtype != torch.bfloat16 or len(shape) != 3:
        raise TypeError(f"{name} must be bfloat16, [tokens, heads, head_dim]")
    T, h, d = shape
    if (stride[2] != 1 and d > 1) or (stride[1] != d and h > 1):
        raise ValueError(f"the heads of a token of {name} must lie side by side")
    return stride[0] if T > 1 else h * d


def _covers(off, T):
    """Do the examples cover all tokens? (Read at the addresses of the first and last offset: indexing a tensor takes microseconds.)"""
    at = off.data_ptr()
    return C.c_int64.from_address(at).value == 0 and C.c_int64.from_address(at + 8 * (off.numel() - 1)).value == T


def _heads_like(t, whole, stream):
    """A new bf16 output of t's shape; zeros where the examples leave tokens out, whose rows no kernel writes."""
    T, h, d = t.shape
    if stream is None:
        out = torch.empty_strided((T, h, d), (h * d, d, 1), dtype=torch.bfloat16, device=t.device)
    else:
        out = _new((T, h, d), torch.bfloat16, t.device, stream)
    return out if whole else _zeroed(out, stream)


def _zeroed(t, stream):
    if _elsewhere(stream):
        with torch.cuda.stream(stream):
            t.zero_()
    else:
        t.zero_()
    return t


def qless_attention_workspace(tokens, n, heads, kv_heads):
    return int(lib().qless_attention_workspace(tokens, n, heads, kv_heads))


def qless_attention_backward_workspace(tokens, n, heads, kv_heads):
    return int(lib().qless_attention_backward_workspace(tokens, n, heads, kv_heads))


def _heads_of(q, k, v):
    T, heads, d = q.shape
    if k.shape != v.shape or k.dim() != 3 or k.shape[0] != T or k.shape[2] != d:
        raise ValueError("shapes of q, k and v do not fit together")
    return T, heads, k.shape[1], d


def qless_attention(q, k, v, offsets, scale=None, out=None, workspace=None, stream=None):
    """Causal attention over packed examples with grouped heads: q bf16 [tokens, heads, head_dim], k, v bf16 [tokens, kv_heads, head_dim] (a
    stride between tokens is allowed); offsets: int64 CPU tensor (or sequence) [n + 1] of the examples' first tokens; scale: head_dim ** -0.5
    by default. Returns dict(out bf16 [tokens, heads, head_dim], lse f32 [tokens, heads]). Rows outside the examples are left as they are
    in a given `out` and are zeros in a new one."""
    off = _host_offsets(offsets)
    sq, sk, sv = _token_stride(q, "q"), _token_stride(k, "k"), _token_stride(v, "v")
    T, heads, kv, d = _heads_of(q, k, v)
    n = off.numel() - 1
    at = _on_gpu(stream, q, k, v, out, workspace)
    whole = _covers(off, T)
    if out is None:
        out, so = _heads_like(q, whole, stream), heads * d
    elif out.shape != q.shape:
        raise ValueError("out must have q's shape")
    else:
        so = _token_stride(out, "out")
    lse = _empty(T, heads, torch.float32, q.device, stream)
    if not whole:
        _zeroed(lse, stream)
    ws, ws_bytes, _hold = _workspace_if(lib().qless_attention_workspace(T, n, heads, kv), q.device, workspace, stream)
    if stream is not None:
        _used(stream, q, k, v, out, workspace)
    _check(lib().qless_attention(q.data_ptr(), sq, k.data_ptr(), sk, v.data_ptr(), sv, off.data_ptr(), T, n, heads, kv, d,
                                 d ** -0.5 if scale is None else scale, out.data_ptr(), so, lse.data_ptr(), ws, ws_bytes,
                                 _stream(stream, at)))
    return dict(out=out, lse=lse)


def qless_attention_backward(grad_out, q, k, v, out, lse, offsets, scale=None, grads=None, workspace=None, stream=None):
    """Gradients of qless_attention from the out and lse that it returned. Returns dict(grad_q, grad_k, grad_v), bf16, of the shapes of q, k
    and v. `grads` may pass preallocated tensors by those names (slices of one matrix, say); rows outside the examples are left as they are in
    those and are zeros in new ones."""
    off = _host_offsets(offsets)
    sg, sq, sk, sv, so = _token_stride(grad_out, "grad_out"), _token_stride(q, "q"), _token_stride(k, "k"), _token_stride(v, "v"), _token_stride(out, "out")
    T, heads, kv, d = _heads_of(q, k, v)
    if grad_out.shape != q.shape or out.shape != q.shape:
        raise ValueError("grad_out and out must have q's shape")
    if lse.shape != (T, heads) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be contiguous float32, [tokens, heads]")
    n = off.numel() - 1
    whole = _covers(off, T)
    if grads is None:
        at = _on_gpu(stream, q, k, v, grad_out, out, lse, workspace)
        gq, gk, gv = _heads_like(q, whole, stream), _heads_like(k, whole, stream), _heads_like(v, whole, stream)
        tq, tk, tv = heads * d, kv * d, kv * d
    else:
        at = _on_gpu(stream, q, k, v, grad_out, out, lse, workspace, *grads.values())
        got = []
        for name, like in (("grad_q", q), ("grad_k", k), ("grad_v", v)):
            t = grads.get(name)
            if t is None:
                t = _heads_like(like, whole, stream)
            elif t.shape != like.shape:
                raise ValueError(f"{name} has the wrong shape")
            got.append(t)
        gq, gk, gv = got
        tq, tk, tv = _token_stride(gq, "grad_q"), _token_stride(gk, "grad_k"), _token_stride(gv, "grad_v")
    ws, ws_bytes, _hold = _workspace_if(lib().qless_attention_backward_workspace(T, n, heads, kv), q.device, workspace, stream)
    if stream is not None:
        _used(stream, q, k, v, grad_out, out, lse, workspace, gq, gk, gv)
    _check(lib().qless_attention_backward(grad_out.data_ptr(), sg, q.data_ptr(), sq, k.data_ptr(), sk, v.data_ptr(), sv, out.data_ptr(), so, lse.data_ptr(),
                                          off.data_ptr(), T, n, heads, kv, d, d ** -0.5 if scale is None else scale, gq.data_ptr(), tq, gk.data_ptr(), tk,
                                          gv.data_ptr(), tv, ws, ws_bytes, _stream(stream, at)))
    return dict(grad_q=gq, grad_k=gk, grad_v=gv)


def _activation_code(activation):
    if activation not in ("silu", "gelu"):
        raise ValueError("activation must be 'silu' or 'gelu'")
    return SILU if activation == "silu" else GELU


def _ffn_shapes(x, w_gate, w_up, w_down):
    inner, width = w_gate.shape
    if x.dim() != 2 or x.shape[1] != width or w_up.shape != (inner, width) or w_down.shape != (width, inner):
        raise ValueError("shapes of the tokens, w_gate, w_up and w_down do not fit together")
    return x.shape[0], width, inner


def _bf16(t):
    if t.dtype != torch.bfloat16:
        raise TypeError("matrices must be bfloat16")
    return t.data_ptr()


def _bf16_args(*tensors):
    """Pointer and row stride of each bf16 matrix (None: absent)."""
    args = []
    for t in tensors:
        if t is None:
            args += [None, 0]
            continue
        args += [_bf16(t), _row_stride(t)]
    return args


def _outputs(given, wanted, device, stream):
    """name -> [rows, cols] bf16: the caller's tensor of that name or a new one (None where it is neither given nor wanted)."""
    given = given or {}
    got = {}
    for name, (want, rows, cols) in wanted.items():
        t = given.get(name)
        if t is None:
            t = _empty(rows, cols, torch.bfloat16, device, stream) if want else None
        elif t.shape != (rows, cols) or t.dtype != torch.bfloat16:
            raise ValueError(f"{name} has the wrong shape or type")
        got[name] = t
    return got


def qless_gated_ffn_workspace(tokens, width, inner):
    return int(lib().qless_gated_ffn_workspace(tokens, width, inner))


def qless_gated_ffn_backward_workspace(tokens, width, inner, want_weight=False):
    return int(lib().qless_gated_ffn_backward_workspace(tokens, width, inner, 1 if want_weight else 0))


def qless_gated_ffn(x, w_gate, w_up, w_down, activation="silu", want_saved=False, out=None, workspace=None, stream=None):
    """Gated feed-forward block out = (act(x w_gate^T) * (x w_up^T)) w_down^T: x bf16 [tokens, width], w_gate, w_up bf16 [inner, width], w_down
    bf16 [width, inner]; activation 'silu' or 'gelu'. Returns dict(out [tokens, width], hidden [tokens, inner]: the down projection's
    input, gate, up [tokens, inner] | None: kept for the backward pass where want_saved). `out` may pass preallocated tensors by those names."""
    T, width, inner = _ffn_shapes(x, w_gate, w_up, w_down)
    code = _activation_code(activation)
    gate = up = None
    if out is None:
        at = _on_gpu(stream, x, w_gate, w_up, w_down, workspace)
        dev = x.device
        y, hidden = _empty(T, width, torch.bfloat16, dev, stream), _empty(T, inner, torch.bfloat16, dev, stream)
        if want_saved:
            gate, up = _empty(T, inner, torch.bfloat16, dev, stream), _empty(T, inner, torch.bfloat16, dev, stream)
    else:
        at = _on_gpu(stream, x, w_gate, w_up, w_down, workspace, *out.values())
        keep = want_saved or out.get("gate") is not None or out.get("up") is not None
        got = _outputs(out, dict(out=(True, T, width), hidden=(True, T, inner), gate=(keep, T, inner), up=(keep, T, inner)), x.device, stream)
        y, hidden, gate, up = got["out"], got["hidden"], got["gate"], got["up"]
    ws, ws_bytes, _hold = _workspace_if(lib().qless_gated_ffn_workspace(T, width, inner), x.device, workspace, stream)
    if stream is not None:
        _used(stream, x, w_gate, w_up, w_down, workspace, y, hidden, gate, up)
    _check(lib().qless_gated_ffn(_bf16(x), _row_stride(x), _bf16(w_gate), _row_stride(w_gate), _bf16(w_up), _row_stride(w_up), _bf16(w_down), _row_stride(w_down),
                                 T, width, inner, code, _bf16(y), _row_stride(y), _bf16(hidden), _row_stride(hidden), *_bf16_args(gate, up), ws, ws_bytes,
                                 _stream(stream, at)))
    return dict(out=y, hidden=hidden, gate=gate, up=up)


def qless_gated_ffn_backward(grad_out, x, gate, up, w_gate, w_up, w_down, activation="silu", want_x=True, want_weight=False, grads=None,
                             workspace=None, stream=None):
    """Gradients of qless_gated_ffn from the gate and up that it kept. Returns dict(grad_x [tokens, width] | None, grad_gate, grad_up [tokens, inner]: at
    the two projections' outputs, grad_w_gate, grad_w_up, grad_w_down | None: where want_weight). `grads` may pass preallocated
    tensors by those names. x may be None where no weight's gradient is wanted."""
    T, width, inner = _ffn_shapes(grad_out, w_gate, w_up, w_down)
    code = _activation_code(activation)
    if gate.shape != (T, inner) or up.shape != (T, inner) or (x is not None and x.shape != (T, width)):
        raise ValueError("x must be [tokens, width], gate and up [tokens, inner]")
    dev = grad_out.device
    if grads is None:
        at = _on_gpu(stream, grad_out, x, gate, up, w_gate, w_up, w_down, workspace)
        gx = _empty(T, width, torch.bfloat16, dev, stream) if want_x else None
        gg, gu = _empty(T, inner, torch.bfloat16, dev, stream), _empty(T, inner, torch.bfloat16, dev, stream)
        wg = wu = wd = None
        if want_weight:
            wg, wu = _empty(inner, width, torch.bfloat16, dev, stream), _empty(inner, width, torch.bfloat16, dev, stream)
            wd = _empty(width, inner, torch.bfloat16, dev, stream)
    else:
        at = _on_gpu(stream, grad_out, x, gate, up, w_gate, w_up, w_down, workspace, *grads.values())
        got = _outputs(grads, dict(grad_x=(want_x, T, width), grad_gate=(True, T, inner), grad_up=(True, T, inner), grad_w_gate=(want_weight, inner, width),
                                   grad_w_up=(want_weight, inner, width), grad_w_down=(want_weight, width, inner)), dev, stream)
        gx, gg, gu, wg, wu, wd = got.values()
    weights = wg is not None or wu is not None or wd is not None
    ws, ws_bytes, _hold = _workspace_if(lib().qless_gated_ffn_backward_workspace(T, width, inner, 1 if weights else 0), dev, workspace, stream)
    if stream is not None:
        _used(stream, grad_out, x, gate, up, w_gate, w_up, w_down, workspace, gx, gg, gu, wg, wu, wd)
    _check(lib().qless_gated_ffn_backward(*_bf16_args(grad_out, x), _bf16(gate), _row_stride(gate), _bf16(up), _row_stride(up), _bf16(w_gate), _row_stride(w_gate),
                                          _bf16(w_up), _row_stride(w_up), _bf16(w_down), _row_stride(w_down), T, width, inner, code, *_bf16_args(gx),
                                          _bf16(gg), _row_stride(gg), _bf16(gu), _row_stride(gu), *(_bf16_args(wg, wu, wd) if weights else (None, 0) * 3),
                                          ws, ws_bytes, _stream(stream, at)))
    return dict(grad_x=gx, grad_gate=gg, grad_up=gu, grad_w_gate=wg, grad_w_up=wu, grad_w_down=wd)


def qless_set_projection_path(path):
    """0 = tensor-core projection kernel (default), 1 = CUDA-core cross-check kernel."""
    _check(lib().qless_set_projection_path(int(path)))


def qless_selftest_timeout(polls=1024, stream=None):
    """Enqueues the bounded-wait self-test kernel; the next qless_check() on the stream raises ERR_TIMEOUT."""
    _check(lib().qless_selftest_timeout(int(polls), _stream(stream)))


def qless_set_select_path(path):
    """0 = by size (default), 1 = multi-pass select at every N, 2 = sampled bracket forced too high."""
    _check(lib().qless_set_select_path(int(path)))


def qless_set_score_path(path):
    """0 = tensor-core scoring kernel for 8/4/2-bit codes (default), 1 = CUDA-core kernel."""
    _check(lib().qless_set_score_path(int(path)))


MICROBENCH = {"bf16_ss": 0, "bf16_ts": 1, "i8_ss": 2, "bf16_ss_pair": 3, "bf16_ts_pair": 4, "i8_ss_pair": 5, "popc": 6, "i8_ts_pair": 7,
              "i8_ss_pair_n448": 8, "tma_l2_stream": 9, "i8_n448_with_tma": 10, "i8_n448_commit_per_block": 11, "i8_n448_streamed_operands": 12,
              "fp4_ss_pair_n448": 13, "fp4_ts_pair": 14}


def qless_microbench(what, iters, device="cuda", stream=None, scratch=None):
    """(milliseconds, operations) of one peak-rate micro-benchmark; `what` is a key of MICROBENCH. `scratch`: a
    uint8 device tensor of at least 4 MiB whose contents the streaming benchmarks read (default: uninitialised)."""
    ms, ops = C.c_float(0), C.c_double(0)
    if scratch is None:
        scratch = _new(4 << 20, torch.uint8, device, stream)
    _check(lib().qless_microbench(MICROBENCH[what], int(iters), C.byref(ms), C.byref(ops), _ptr(scratch), scratch.numel(),
                                  _stream(stream)))
    return ms.value, ops.value
