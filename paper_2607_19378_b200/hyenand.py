"""ctypes binding of libhyenand.so: argument marshalling only.

Every function has the name and meaning of the C entry point declared in
include/hyenand.h; tensors are passed as raw device (or host) pointers and all
arithmetic happens in the library's CUDA kernels.  There is no fallback: if the
library has not been built, loading raises.  Recurrence, DeltaRule, Heads, Block and Dropout marshal
their arguments in a compiled module (csrc/calls.cpp).
"""
from __future__ import annotations

import ctypes
import functools
import importlib.machinery
import importlib.util
import math
import os

import torch

from .build import calls_path

_HERE = os.path.dirname(os.path.abspath(__file__))
# HYENAND_LIB=debug selects the checked build (libhyenand_debug.so, see hyenand_debug_build in the header)
LIB_PATH = os.path.join(_HERE, "libhyenand_debug.so" if os.environ.get("HYENAND_LIB") == "debug" else "libhyenand.so")

HYENAND_F32 = 0
HYENAND_BF16 = 1
HYENAND_MODE_LINEAR = 0
HYENAND_MODE_CAUSAL = 1
HYENAND_MODE_CIRCULAR = 2
HYENAND_DECAY_VALUE = 0
HYENAND_DECAY_LOG = 1
HYENAND_DECAY_SIGMOID = 2
HYENAND_DECAY_NONE = 3
HYENAND_NORM_NONE = 0
HYENAND_NORM_RMS = 1
HYENAND_NORM_L2 = 2
HYENAND_GATE_NONE = 0
HYENAND_GATE_SIGMOID = 1
HYENAND_GATE_SILU = 2
HYENAND_OK = 0
HYENAND_ERR_INVALID_ARG = 1
HYENAND_ERR_UNSUPPORTED = 2
HYENAND_ERR_ALLOC = 3
HYENAND_ERR_CUDA = 4

_DTYPES = {torch.float32: HYENAND_F32, torch.bfloat16: HYENAND_BF16}
_lib = None


class HyenaNDError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"hyenand error {code}: {msg}")
        self.code = code


def lib() -> ctypes.CDLL:
    """The loaded C library (raises if it was never built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_19378_b200.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, ip, ll = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int), ctypes.c_longlong
        L.hyenand_create_plan.restype = vp
        L.hyenand_create_plan.argtypes = [ctypes.c_int, ip, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.hyenand_create_plan_mode.restype = vp
        L.hyenand_create_plan_mode.argtypes = [ctypes.c_int, ip, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.hyenand_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        L.hyenand_forward_ex.argtypes = [vp, vp, vp, vp, vp, ll, vp, vp]
        L.hyenand_forward_host.argtypes = [vp, vp, vp, vp, vp, ll, vp, vp]
        L.hyenand_destroy_plan.argtypes = [vp]
        L.hyenand_destroy_plan.restype = None
        L.hyenand_last_error.restype = ctypes.c_char_p
        L.hyenand_debug_build.restype = ctypes.c_int
        L.hyenand_debug_violations.restype = ll
        L.hyenand_debug_violations.argtypes = [ctypes.POINTER(ctypes.c_ulonglong), ip, ctypes.POINTER(ctypes.c_char_p)]
        L.hyenand_debug_selftest.restype = ll
        L.hyenand_synth_device_status.restype = ctypes.c_int
        L.hyenand_selftest_bounded_wait.argtypes = [ctypes.c_int]
        L.hyenand_selftest_bounded_wait.restype = ctypes.c_int
        L.hyenand_plan_device_status.argtypes = [vp]
        L.hyenand_plan_device_status.restype = ctypes.c_int
        L.hyenand_plan_workspace_bytes.argtypes = [vp]
        L.hyenand_plan_workspace_bytes.restype = ctypes.c_size_t
        L.hyenand_plan_fft_dims.argtypes = [vp, ip]
        L.hyenand_plan_launches.argtypes = [vp, ctypes.c_int]
        L.hyenand_plan_path.argtypes = [vp]
        L.hyenand_plan_path.restype = ctypes.c_char_p
        L.hyenand_plan_groups.argtypes = [vp, ctypes.POINTER(ll), ip]
        L.hyenand_plan_guard_damage.argtypes = [vp]
        L.hyenand_plan_guard_damage.restype = ll
        dpp = ctypes.POINTER(ctypes.c_double)
        L.hyenand_plan_kernel_count.argtypes = [vp]
        L.hyenand_plan_kernel_info.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_char_p),
                                               dpp, dpp, dpp]
        L.hyenand_noalloc_max_bytes.restype = ctypes.c_size_t
        L.hyenand_forward_noalloc.argtypes = [ctypes.c_int, ip, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                              vp, vp, vp, vp, ll, vp, vp]
        fp = ctypes.POINTER(ctypes.c_float)
        L.hyenand_mixer_create.restype = vp
        L.hyenand_mixer_create.argtypes = [ctypes.c_int, ip, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_float]
        L.hyenand_mixer_forward.argtypes = [vp, vp, vp, vp, vp, ll, vp, vp, vp, vp]
        L.hyenand_mixer_plan.restype = vp
        L.hyenand_mixer_plan.argtypes = [vp]
        L.hyenand_mixer_guard_damage.restype = ll
        L.hyenand_mixer_guard_damage.argtypes = [vp]
        L.hyenand_mixer_destroy.restype = None
        L.hyenand_mixer_destroy.argtypes = [vp]
        L.hyenand_backward_create.restype = vp
        L.hyenand_backward_create.argtypes = [ctypes.c_int, ip, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.hyenand_backward.argtypes = [vp, vp, vp, vp, vp, ll, vp, vp, vp, vp, vp, vp]
        L.hyenand_backward_guard_damage.restype = ll
        L.hyenand_backward_guard_damage.argtypes = [vp]
        L.hyenand_backward_destroy.restype = None
        L.hyenand_backward_destroy.argtypes = [vp]
        L.hyenand_synthesize_kernel.argtypes = [ctypes.c_int, ip] + [ctypes.c_int] * 5 + [vp] * 10 + [ctypes.c_int, vp, vp]
        ci, cf = ctypes.c_int, ctypes.c_float
        L.hyenand_recurrence_marks.restype = ll
        L.hyenand_recurrence_marks.argtypes = [ci]
        L.hyenand_recurrence_forward.argtypes = [ci] * 5 + [vp] * 11
        L.hyenand_recurrence_backward.argtypes = [ci] * 5 + [vp] * 15
        L.hyenand_recurrence_workspace_bytes.restype = ll
        L.hyenand_recurrence_workspace_bytes.argtypes = [ci] * 4
        L.hyenand_recurrence_step.argtypes = [ci] * 4 + [vp] * 9
        L.hyenand_delta_marks.restype = ll
        L.hyenand_delta_marks.argtypes = [ci] * 3
        L.hyenand_delta_workspace_bytes.restype = ll
        L.hyenand_delta_workspace_bytes.argtypes = [ci] * 8
        L.hyenand_delta_forward.argtypes = [ci] * 8 + [vp] * 12
        L.hyenand_delta_backward.argtypes = [ci] * 8 + [vp] * 17
        L.hyenand_delta_step.argtypes = [ci] * 7 + [vp] * 10
        L.hyenand_heads_workspace_bytes.restype = ll
        L.hyenand_heads_workspace_bytes.argtypes = [ci, ip] + [ci] * 5
        L.hyenand_heads_forward.argtypes = [ci, ip] + [ci] * 6 + [ip, ctypes.c_double, ctypes.c_float] + [vp] * 8
        L.hyenand_heads_backward.argtypes = [ci, ip] + [ci] * 6 + [ip, ctypes.c_double, ctypes.c_float] + [vp] * 13
        L.hyenand_block_workspace_bytes.restype = ll
        L.hyenand_block_workspace_bytes.argtypes = [ci] * 4
        L.hyenand_block_forward.argtypes = [ci] * 4 + [vp] * 6 + [cf, ci, cf, vp, ci] + [vp] * 4
        L.hyenand_block_backward.argtypes = [ci] * 4 + [vp] * 6 + [cf, ci, cf, vp, ci] + [vp] * 11
        L.hyenand_dropout.argtypes = [ll, ci, vp, cf, vp, ci, vp, vp]
        L.hyenand_plan_set_timing.argtypes = [vp, ctypes.c_int]
        L.hyenand_plan_kernel_time.argtypes = [vp, ctypes.c_int, dpp, dpp]
        _lib = L
    return _lib


def hyenand_last_error() -> str:
    return lib().hyenand_last_error().decode()


def hyenand_last_error_code() -> int:
    return int(lib().hyenand_last_error_code())


def _check(code: int):
    if code != HYENAND_OK:
        raise HyenaNDError(code, hyenand_last_error())


def hyenand_create_plan(ndim: int, dims, B: int, C: int, causal: int, dtype: int) -> int:
    arr = _dims_array(tuple(map(int, dims)))
    h = lib().hyenand_create_plan(int(ndim), arr, int(B), int(C), int(causal), int(dtype))
    if not h:
        msg = hyenand_last_error()
        code = hyenand_last_error_code() or HYENAND_ERR_INVALID_ARG
        raise HyenaNDError(code, msg)
    return h


def hyenand_create_plan_mode(ndim: int, dims, B: int, C: int, mode: int, dtype: int) -> int:
    arr = _dims_array(tuple(map(int, dims)))
    h = lib().hyenand_create_plan_mode(int(ndim), arr, int(B), int(C), int(mode), int(dtype))
    if not h:
        msg = hyenand_last_error()
        code = hyenand_last_error_code() or HYENAND_ERR_INVALID_ARG
        raise HyenaNDError(code, msg)
    return h


def hyenand_destroy_plan(plan: int) -> None:
    lib().hyenand_destroy_plan(plan)


@functools.lru_cache(maxsize=64)
def _dims_array(dims: tuple):
    """dims as a C int array (read only: the library copies what it keeps)."""
    return (ctypes.c_int * max(1, len(dims)))(*dims)


# The calls below are the launch path of small problems, whose kernels take a few microseconds: no tensor views, no stream
# objects, shapes compared with tuples worked out when the object was created (one 32x32x8 forward: 15.2 us a call when the
# filter's stride came from h[0, 0].numel() and the stream from torch.cuda.current_stream(), 8 now).

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def hyenand_forward(plan: int, q, k, v, h, y, stream=None) -> None:
    _check(lib().hyenand_forward(plan, q.data_ptr(), k.data_ptr(), v.data_ptr(), h.data_ptr(),
                                 y.data_ptr(), _stream_ptr(stream)))


def hyenand_forward_ex(plan: int, q, k, v, h, h_batch_stride_elems: int, y, stream=None) -> None:
    _check(lib().hyenand_forward_ex(plan, q.data_ptr(), k.data_ptr(), v.data_ptr(), h.data_ptr(),
                                    int(h_batch_stride_elems), y.data_ptr(), _stream_ptr(stream)))


def hyenand_forward_host(plan: int, q, k, v, h, h_batch_stride_elems: int, y, stream=None) -> None:
    _check(lib().hyenand_forward_host(plan, q.data_ptr(), k.data_ptr(), v.data_ptr(), h.data_ptr(),
                                      int(h_batch_stride_elems), y.data_ptr(), _stream_ptr(stream)))


def hyenand_debug_build() -> bool:
    return bool(lib().hyenand_debug_build())


def hyenand_debug_violations():
    """(count, first address, first line, first file) of the checked build's out-of-range accesses since the last call;
    count is -1 in the product library."""
    addr, line, name = ctypes.c_ulonglong(), ctypes.c_int(), ctypes.c_char_p()
    n = lib().hyenand_debug_violations(ctypes.byref(addr), ctypes.byref(line), ctypes.byref(name))
    return int(n), int(addr.value), int(line.value), (name.value or b"").decode()


def hyenand_synth_device_status() -> int:
    return int(lib().hyenand_synth_device_status())


def hyenand_debug_selftest() -> int:
    return int(lib().hyenand_debug_selftest())


def hyenand_selftest_bounded_wait(polls: int = 1000) -> int:
    """9 if a wait on a barrier that nothing completes ran out and was reported, as it must."""
    return int(lib().hyenand_selftest_bounded_wait(int(polls)))


def hyenand_plan_device_status(plan: int) -> int:
    """0 unless a kernel of the plan gave up a bounded wait (synchronise the stream first)."""
    return int(lib().hyenand_plan_device_status(plan))


def hyenand_plan_workspace_bytes(plan: int) -> int:
    return int(lib().hyenand_plan_workspace_bytes(plan))


def hyenand_plan_fft_dims(plan: int, ndim: int):
    out = (ctypes.c_int * ndim)()
    _check(lib().hyenand_plan_fft_dims(plan, out))
    return tuple(out)


def hyenand_plan_launches(plan: int, h_shared: bool) -> int:
    return int(lib().hyenand_plan_launches(plan, 1 if h_shared else 0))


def hyenand_plan_path(plan: int) -> str:
    return lib().hyenand_plan_path(plan).decode()


def hyenand_plan_groups(plan: int):
    """(slices per group, lanes): how one forward schedules the batch."""
    n, lanes = ctypes.c_longlong(), ctypes.c_int()
    _check(lib().hyenand_plan_groups(plan, ctypes.byref(n), ctypes.byref(lanes)))
    return int(n.value), int(lanes.value)


def hyenand_plan_guard_damage(plan: int) -> int:
    """Bytes of the guard bands around the plan's device allocations that a kernel overwrote (0 = none)."""
    return int(lib().hyenand_plan_guard_damage(plan))


def hyenand_plan_kernel_count(plan: int) -> int:
    return int(lib().hyenand_plan_kernel_count(plan))


def hyenand_plan_kernel_info(plan: int, kernel_id: int, h_shared: bool):
    """(name, launches, algorithmic bytes, algorithmic flops) of one kernel, per forward."""
    name = ctypes.c_char_p()
    n, b, f = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    _check(lib().hyenand_plan_kernel_info(plan, kernel_id, 1 if h_shared else 0, ctypes.byref(name),
                                          ctypes.byref(n), ctypes.byref(b), ctypes.byref(f)))
    return name.value.decode(), n.value, b.value, f.value


def hyenand_plan_set_timing(plan: int, enable) -> None:
    """0/False: off; 1/True: time every launch; 2: the same with the plan's lanes run one after the other."""
    _check(lib().hyenand_plan_set_timing(plan, int(enable)))


def hyenand_plan_kernel_time(plan: int, kernel_id: int):
    """(accumulated device ms, recorded launches) since timing was switched on."""
    ms, n = ctypes.c_double(), ctypes.c_double()
    _check(lib().hyenand_plan_kernel_time(plan, kernel_id, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def hyenand_noalloc_max_bytes() -> int:
    return int(lib().hyenand_noalloc_max_bytes())


def hyenand_forward_noalloc(dims, B: int, C: int, causal: int, dtype: int, q, k, v, h,
                            h_batch_stride_elems: int, y, stream=None) -> None:
    """Forward through the entry point that allocates no device memory (fixed workspace inside
    the library; see include/hyenand.h for its limits and the rule about overlapping calls)."""
    arr = _dims_array(tuple(map(int, dims)))
    _check(lib().hyenand_forward_noalloc(len(dims), arr, int(B), int(C), int(causal), int(dtype),
                                         q.data_ptr(), k.data_ptr(), v.data_ptr(), h.data_ptr(),
                                         int(h_batch_stride_elems), y.data_ptr(), _stream_ptr(stream)))


def hyenand_mixer_create(ndim: int, dims, B: int, C: int, mode: int, dtype: int, eps: float) -> int:
    arr = _dims_array(tuple(map(int, dims)))
    h = lib().hyenand_mixer_create(int(ndim), arr, int(B), int(C), int(mode), int(dtype), float(eps))
    if not h:
        raise HyenaNDError(hyenand_last_error_code() or HYENAND_ERR_INVALID_ARG, hyenand_last_error())
    return h


def hyenand_mixer_forward(mixer: int, q, k, v, h, h_batch_stride_elems: int, g_in, g_out, y, stream=None) -> None:
    _check(lib().hyenand_mixer_forward(mixer, q.data_ptr(), k.data_ptr(), v.data_ptr(), h.data_ptr(),
                                       int(h_batch_stride_elems), g_in.data_ptr(), g_out.data_ptr(), y.data_ptr(),
                                       _stream_ptr(stream)))


def hyenand_mixer_plan(mixer: int) -> int:
    return lib().hyenand_mixer_plan(mixer)


def hyenand_mixer_guard_damage(mixer: int) -> int:
    return int(lib().hyenand_mixer_guard_damage(mixer))


def hyenand_mixer_destroy(mixer: int) -> None:
    lib().hyenand_mixer_destroy(mixer)


def hyenand_synthesize_kernel(dims, mode: int, B: int, C: int, hidden: int, layers: int, W1, b1, omega0, Wh, bh, Wout,
                              bout, gamma, beta, window, dtype: int, h, stream=None) -> None:
    """K(x) on the tap grid of `dims` into h (device tensor [B, C, K..]); parameters: fp32 device tensors, gamma and
    beta may both be None (static kernel), Wh and bh may be None when layers == 1."""
    arr = _dims_array(tuple(map(int, dims)))
    ptr = lambda t: None if t is None else t.data_ptr()
    _check(lib().hyenand_synthesize_kernel(len(dims), arr, int(mode), int(B), int(C), int(hidden), int(layers),
                                           ptr(W1), ptr(b1), ptr(omega0), ptr(Wh), ptr(bh), ptr(Wout), ptr(bout),
                                           ptr(gamma), ptr(beta), ptr(window), int(dtype), h.data_ptr(), _stream_ptr(stream)))


def hyenand_backward_create(ndim: int, dims, B: int, C: int, mode: int, dtype: int) -> int:
    arr = _dims_array(tuple(map(int, dims)))
    h = lib().hyenand_backward_create(int(ndim), arr, int(B), int(C), int(mode), int(dtype))
    if not h:
        raise HyenaNDError(hyenand_last_error_code() or HYENAND_ERR_INVALID_ARG, hyenand_last_error())
    return h


def hyenand_backward(grad: int, q, k, v, h, h_batch_stride_elems: int, dy, dq, dk, dv, dh, stream=None) -> None:
    _check(lib().hyenand_backward(grad, q.data_ptr(), k.data_ptr(), v.data_ptr(), h.data_ptr(), int(h_batch_stride_elems),
                                  dy.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dh.data_ptr(), _stream_ptr(stream)))


def hyenand_backward_guard_damage(grad: int) -> int:
    return int(lib().hyenand_backward_guard_damage(grad))


def hyenand_backward_destroy(grad: int) -> None:
    lib().hyenand_backward_destroy(grad)


def _ptr(t):
    return None if t is None else t.data_ptr()


def hyenand_recurrence_marks(L: int) -> int:
    return int(lib().hyenand_recurrence_marks(int(L)))


def hyenand_recurrence_workspace_bytes(B: int, C: int, L: int, dtype: int) -> int:
    return int(lib().hyenand_recurrence_workspace_bytes(B, C, L, dtype))


def hyenand_recurrence_device_status() -> int:
    return int(lib().hyenand_recurrence_device_status())


def _ints(values):
    """A C array of int; what does not fit in one is refused, not cut off."""
    if any(not -(1 << 31) <= int(n) < 1 << 31 for n in values):
        raise OverflowError("a size must fit in 32 bits")
    return (ctypes.c_int * len(values))(*(int(n) for n in values))


def hyenand_delta_marks(L: int, Dk: int, Dv: int) -> int:
    return int(lib().hyenand_delta_marks(*_ints((L, Dk, Dv))))


def hyenand_delta_workspace_bytes(B: int, H: int, Hk: int, L: int, Dk: int, Dv: int, dtype: int, backward: int) -> int:
    return int(lib().hyenand_delta_workspace_bytes(*_ints((B, H, Hk, L, Dk, Dv, dtype, backward))))


def hyenand_delta_device_status() -> int:
    return int(lib().hyenand_delta_device_status())


def hyenand_debug_delta_late(kernel: int, chunk: int = 0, wait: int = 0) -> int:
    return int(lib().hyenand_debug_delta_late(int(kernel), int(chunk), int(wait)))


def hyenand_delta_forward(B: int, H: int, Hk: int, L: int, Dk: int, Dv: int, decay: int, dtype: int, q, k, v, g, beta, s0, lengths, y, s_end, marks,
                          workspace, stream=None) -> None:
    _check(lib().hyenand_delta_forward(*_ints((B, H, Hk, L, Dk, Dv, decay, dtype)), q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(g), beta.data_ptr(),
                                       _ptr(s0), _ptr(lengths), y.data_ptr(), _ptr(s_end), _ptr(marks), workspace.data_ptr(), _stream_ptr(stream)))


def hyenand_delta_backward(B: int, H: int, Hk: int, L: int, Dk: int, Dv: int, decay: int, dtype: int, q, k, v, g, beta, lengths, marks, dy, ds_end,
                           dq, dk, dv, dg, dbeta, ds0, workspace, stream=None) -> None:
    _check(lib().hyenand_delta_backward(*_ints((B, H, Hk, L, Dk, Dv, decay, dtype)), q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(g), beta.data_ptr(),
                                        _ptr(lengths), marks.data_ptr(), dy.data_ptr(), _ptr(ds_end), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                        _ptr(dg), dbeta.data_ptr(), _ptr(ds0), workspace.data_ptr(), _stream_ptr(stream)))


def hyenand_delta_step(B: int, H: int, Hk: int, Dk: int, Dv: int, decay: int, dtype: int, q, k, v, g, beta, state, active, y, new_state, stream=None) -> None:
    _check(lib().hyenand_delta_step(*_ints((B, H, Hk, Dk, Dv, decay, dtype)), q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(g), beta.data_ptr(),
                                    state.data_ptr(), _ptr(active), y.data_ptr(), new_state.data_ptr(), _stream_ptr(stream)))


def hyenand_heads_workspace_bytes(ndim: int, dims, B: int, Hq: int, Hk: int, D: int, dtype: int) -> int:
    return int(lib().hyenand_heads_workspace_bytes(int(ndim), _ints(dims), *_ints((B, Hq, Hk, D, dtype))))


def hyenand_heads_forward(ndim: int, dims, B: int, Hq: int, Hk: int, D: int, dtype: int, norm: int, axes, base: float, eps: float, q, k, g_q, g_k,
                          positions, q_out, k_out, stream=None) -> None:
    _check(lib().hyenand_heads_forward(int(ndim), _ints(dims), *_ints((B, Hq, Hk, D, dtype, norm)), None if axes is None else _ints(axes), float(base),
                                       float(eps), q.data_ptr(), k.data_ptr(), _ptr(g_q), _ptr(g_k), _ptr(positions), q_out.data_ptr(), k_out.data_ptr(),
                                       _stream_ptr(stream)))


def hyenand_heads_backward(ndim: int, dims, B: int, Hq: int, Hk: int, D: int, dtype: int, norm: int, axes, base: float, eps: float, q, k, g_q, g_k,
                           positions, dq_out, dk_out, dq, dk, dg_q, dg_k, workspace, stream=None) -> None:
    _check(lib().hyenand_heads_backward(int(ndim), _ints(dims), *_ints((B, Hq, Hk, D, dtype, norm)), None if axes is None else _ints(axes), float(base),
                                        float(eps), q.data_ptr(), k.data_ptr(), _ptr(g_q), _ptr(g_k), _ptr(positions), dq_out.data_ptr(), dk_out.data_ptr(),
                                        dq.data_ptr(), dk.data_ptr(), _ptr(dg_q), _ptr(dg_k), _ptr(workspace), _stream_ptr(stream)))


def hyenand_debug_recurrence_late(tile: int, warp: int = -1) -> int:
    return int(lib().hyenand_debug_recurrence_late(int(tile), int(warp)))


def hyenand_recurrence_forward(B: int, C: int, L: int, decay: int, dtype: int, q, k, v, g, s0, lengths, y, s_end, marks, workspace=None,
                               stream=None) -> None:
    _check(lib().hyenand_recurrence_forward(B, C, L, decay, dtype, q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), _ptr(s0),
                                            _ptr(lengths), y.data_ptr(), _ptr(s_end), _ptr(marks), _ptr(workspace), _stream_ptr(stream)))


def hyenand_recurrence_backward(B: int, C: int, L: int, decay: int, dtype: int, q, k, v, g, lengths, marks, dy, ds_end, dq, dk, dv, dg, ds0,
                                workspace=None, stream=None) -> None:
    _check(lib().hyenand_recurrence_backward(B, C, L, decay, dtype, q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), _ptr(lengths),
                                             marks.data_ptr(), dy.data_ptr(), _ptr(ds_end), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                             dg.data_ptr(), _ptr(ds0), _ptr(workspace), _stream_ptr(stream)))


def hyenand_recurrence_step(B: int, C: int, decay: int, dtype: int, q, k, v, g, state, active, y, new_state, stream=None) -> None:
    _check(lib().hyenand_recurrence_step(B, C, decay, dtype, q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), state.data_ptr(),
                                         _ptr(active), y.data_ptr(), new_state.data_ptr(), _stream_ptr(stream)))


def hyenand_block_workspace_bytes(B: int, C: int, T: int, dtype: int) -> int:
    return int(lib().hyenand_block_workspace_bytes(B, C, T, dtype))


def hyenand_block_device_status() -> int:
    return int(lib().hyenand_block_device_status())


def hyenand_block_forward(B: int, C: int, T: int, dtype: int, x, m, z, g_post, scale, g_pre, eps: float, gate: int, p: float, rng, site: int,
                          r, n, stats, stream=None) -> None:
    _check(lib().hyenand_block_forward(B, C, T, dtype, x.data_ptr(), m.data_ptr(), _ptr(z), _ptr(g_post), _ptr(scale), _ptr(g_pre), eps, gate,
                                       p, _ptr(rng), site, r.data_ptr(), _ptr(n), _ptr(stats), _stream_ptr(stream)))


def hyenand_block_backward(B: int, C: int, T: int, dtype: int, x, m, z, g_post, scale, g_pre, eps: float, gate: int, p: float, rng, site: int,
                           stats, dr, dn, dx, dm, dz, dg_post, dscale, dg_pre, workspace, stream=None) -> None:
    _check(lib().hyenand_block_backward(B, C, T, dtype, x.data_ptr(), m.data_ptr(), _ptr(z), _ptr(g_post), _ptr(scale), _ptr(g_pre), eps, gate,
                                        p, _ptr(rng), site, _ptr(stats), _ptr(dr), _ptr(dn), dx.data_ptr(), dm.data_ptr(), _ptr(dz),
                                        _ptr(dg_post), _ptr(dscale), _ptr(dg_pre), workspace.data_ptr(), _stream_ptr(stream)))


def hyenand_dropout(n: int, dtype: int, x, p: float, rng, site: int, y, stream=None) -> None:
    _check(lib().hyenand_dropout(n, dtype, x.data_ptr(), p, rng.data_ptr(), site, y.data_ptr(), _stream_ptr(stream)))


def _check_tensors(tensors, dtype, what):
    for t in tensors:
        if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype):
            raise ValueError(f"inputs must be contiguous CUDA tensors of the {what}'s dtype")


class _FilterShape:
    """h's shape -> batch stride: 0 for one filter per channel [C, K..], C K.. for one per sample [B, C, K..]."""

    def __init__(self, B, C, taps):
        self.shared, self.full = (C,) + taps, (B, C) + taps
        self.stride = C
        for K in taps:
            self.stride *= K

    def __call__(self, h) -> int:
        shape = h.shape
        if shape == self.full:
            return self.stride
        if shape == self.shared:
            return 0
        raise ValueError(f"h has shape {tuple(shape)}")


class Backward:
    """Owner of a hyenand_grad handle: dq, dk, dv, dh of the gated long convolution."""

    def __init__(self, dims, B: int, C: int, mode: str = "linear", dtype=torch.float32):
        self.dims = tuple(int(d) for d in dims)
        self.B, self.C, self.mode, self.dtype = B, C, mode, dtype
        code = {"linear": HYENAND_MODE_LINEAR, "causal": HYENAND_MODE_CAUSAL, "circular": HYENAND_MODE_CIRCULAR}[mode]
        self._filter = _FilterShape(B, C, tuple(2 * L - 1 if mode == "linear" else L for L in self.dims))
        self.handle = hyenand_backward_create(len(self.dims), self.dims, B, C, code, _DTYPES[dtype])

    def __call__(self, q, k, v, h, dy, stream=None):
        stride = self._filter(h)
        _check_tensors((q, k, v, h, dy), self.dtype, "handle")
        dq, dk, dv, dh = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q), torch.empty_like(h)
        hyenand_backward(self.handle, q, k, v, h, stride, dy, dq, dk, dv, dh, stream)
        return dq, dk, dv, dh

    def close(self):
        if self.handle:
            hyenand_backward_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Mixer:
    """Owner of a hyenand_mixer handle: the full operator of Eq. 2 (pointwise stages + long convolution)."""

    def __init__(self, dims, B: int, C: int, mode: str = "linear", dtype=torch.float32, eps: float = 1e-6):
        self.dims = tuple(int(d) for d in dims)
        self.B, self.C, self.mode, self.dtype = B, C, mode, dtype
        code = {"linear": HYENAND_MODE_LINEAR, "causal": HYENAND_MODE_CAUSAL, "circular": HYENAND_MODE_CIRCULAR}[mode]
        self._filter = _FilterShape(B, C, tuple(2 * L - 1 if mode == "linear" else L for L in self.dims))
        self.handle = hyenand_mixer_create(len(self.dims), self.dims, B, C, code, _DTYPES[dtype], eps)

    def forward(self, q, k, v, h, g_in, g_out, y=None, stream=None):
        stride = self._filter(h)
        _check_tensors((q, k, v, h), self.dtype, "mixer")
        for g in (g_in, g_out):
            if not (g.is_cuda and g.is_contiguous() and g.dtype == torch.float32 and g.numel() == self.C):
                raise ValueError("g_in, g_out must be contiguous fp32 CUDA tensors of C elements")
        if y is None:
            y = torch.empty_like(q)
        hyenand_mixer_forward(self.handle, q, k, v, h, stride, g_in, g_out, y, stream)
        return y

    def close(self):
        if self.handle:
            hyenand_mixer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Plan:
    """Convenience owner of a plan handle (create on construction, destroy on close)."""

    def __init__(self, dims, B: int, C: int, causal: bool = False, dtype=torch.float32, circular: bool = False):
        self.dims = tuple(int(d) for d in dims)
        self.B, self.C, self.causal, self.dtype, self.circular = B, C, bool(causal), dtype, bool(circular)
        self._stride = _FilterShape(B, C, tuple(L if (self.causal or self.circular) else 2 * L - 1 for L in self.dims))
        if self.circular:
            if self.causal:
                raise ValueError("a plan is causal or circular, not both")
            self.handle = hyenand_create_plan_mode(len(self.dims), self.dims, B, C, HYENAND_MODE_CIRCULAR, _DTYPES[dtype])
        else:
            self.handle = hyenand_create_plan(len(self.dims), self.dims, B, C, int(self.causal), _DTYPES[dtype])

    def forward(self, q, k, v, h, y=None, stream=None):
        """Device tensors in, device tensor out (enqueued on the current stream)."""
        _check_tensors((q, k, v, h), self.dtype, "plan")
        if y is None:
            y = torch.empty_like(q)
        hyenand_forward_ex(self.handle, q, k, v, h, self._stride(h), y, stream)
        return y

    def forward_host(self, q, k, v, h, y, stream=None):
        """Host tensors in, host tensor out; copies run inside the call."""
        hyenand_forward_host(self.handle, q, k, v, h, self._stride(h), y, stream)
        return y

    @property
    def launches_per_forward(self):
        return lambda shared: hyenand_plan_launches(self.handle, shared)

    def close(self):
        if self.handle:
            hyenand_destroy_plan(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _pool(stream):
    """Outputs and workspaces belong to the stream that the kernels run on, as the allocator sees it."""
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


@functools.lru_cache(maxsize=1)
def _calls():
    """The compiled side of the classes below (csrc/calls.cpp); raises if it was never built."""
    path, name = calls_path(), __package__ + "._calls"
    try:
        spec = importlib.util.spec_from_file_location(name, path, loader=importlib.machinery.ExtensionFileLoader(name, path))
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError as e:
        raise OSError(f"{path} cannot be loaded ({e}): build it with `python -m paper_2607_19378_b200.build`") from e
    return module


def _address(name: str) -> int:
    return ctypes.cast(getattr(lib(), name), ctypes.c_void_p).value


class Recurrence:
    """The gated linear recurrence s_t = a_t s_{t-1} + k_t v_t, y_t = q_t s_t on [B, C, L], with a_t = g_t ("value"), exp(g_t)
    ("log") or sigmoid(g_t) ("sigmoid").  Holds the shape only: every call stands for itself, on any stream."""

    def __init__(self, L: int, B: int, C: int, decay: str = "log", dtype=torch.float32):
        self.L, self.B, self.C, self.decay, self.dtype = int(L), int(B), int(C), decay, dtype
        code = {"value": HYENAND_DECAY_VALUE, "log": HYENAND_DECAY_LOG, "sigmoid": HYENAND_DECAY_SIGMOID}[decay]
        marks = hyenand_recurrence_marks(self.L)
        if min(self.B, self.C, marks) < 1:
            raise ValueError("B and C must be >= 1, L between 1 and 2^30")
        self._ops = _calls()
        self._handle = self._ops.make_recurrence(self.B, self.C, self.L, marks, code, _DTYPES[dtype],
                                                 hyenand_recurrence_workspace_bytes(self.B, self.C, self.L, _DTYPES[dtype]),
                                                 _address("hyenand_recurrence_forward"), _address("hyenand_recurrence_backward"), _address("hyenand_recurrence_step"), _check)

    def forward(self, q, k, v, g, s0=None, lengths=None, marks: bool = False, y=None, stream=None):
        """(y, state behind the row), and with marks=True what `backward` needs of this call as a third."""
        if stream is not None:
            with _pool(stream):
                return self.forward(q, k, v, g, s0, lengths, marks, y)
        return self._ops.recurrence_forward(self._handle, q, k, v, g, s0, lengths, marks, y)

    def backward(self, q, k, v, g, marks, dy, ds_end=None, lengths=None, stream=None):
        """dq, dk, dv, dg and ds0, from the marks of a forward call on the same q, k, v, g, s0 and lengths."""
        if stream is not None:
            with _pool(stream):
                return self.backward(q, k, v, g, marks, dy, ds_end, lengths)
        return self._ops.recurrence_backward(self._handle, q, k, v, g, marks, dy, ds_end, lengths)

    def step(self, q, k, v, g, state, new_state=None, active=None, y=None, stream=None):
        """One token: q, k, v, g [B, C] -> y [B, C]; the state is replaced, or left and the new one written to new_state."""
        if stream is not None:
            with _pool(stream):
                return self.step(q, k, v, g, state, new_state, active, y)
        return self._ops.recurrence_step(self._handle, q, k, v, g, state, new_state, active, y)


class DeltaRule:
    """The gated delta rule u_t = beta_t (v_t - a_t S_{t-1} k_t), S_t = a_t S_{t-1} + u_t k_t^T, y_t = S_t q_t on q, k [B, Hk * Dk, L] and
    v [B, H * Dv, L], with a_t = exp(g_t) ("log"), sigmoid(g_t) ("sigmoid") or 1 ("none", g is None); g, beta [B, H, L] fp32, states
    [B, H, Dv, Dk] fp32.  Value head h goes with head h // (H // Hk) of queries and keys.  Holds the shape only: every call stands
    for itself, on any stream."""

    def __init__(self, L: int, B: int, H: int, Dk: int, Dv: int = None, Hk: int = None, decay: str = "log", dtype=torch.float32):
        self.L, self.B, self.H, self.Dk, self.decay, self.dtype = int(L), int(B), int(H), int(Dk), decay, dtype
        self.Dv, self.Hk = self.Dk if Dv is None else int(Dv), self.H if Hk is None else int(Hk)
        code = {"log": HYENAND_DECAY_LOG, "sigmoid": HYENAND_DECAY_SIGMOID, "none": HYENAND_DECAY_NONE}[decay]
        shape = (self.B, self.H, self.Hk, self.L, self.Dk, self.Dv, _DTYPES[dtype])
        work = [hyenand_delta_workspace_bytes(*shape, backward) for backward in (0, 1)]
        if min(work) < 1:
            raise ValueError(hyenand_last_error())
        self._ops = _calls()
        self._handle = self._ops.make_delta(self.B, self.H, self.Hk, self.L, self.Dk, self.Dv, hyenand_delta_marks(self.L, self.Dk, self.Dv), code, _DTYPES[dtype], *work,
                                            _address("hyenand_delta_forward"), _address("hyenand_delta_backward"), _address("hyenand_delta_step"), _check)

    def forward(self, q, k, v, g, beta, s0=None, lengths=None, marks: bool = False, y=None, stream=None):
        """(y, states behind the rows), and with marks=True what `backward` needs of this call as a third."""
        if stream is not None:
            with _pool(stream):
                return self.forward(q, k, v, g, beta, s0, lengths, marks, y)
        return self._ops.delta_forward(self._handle, q, k, v, g, beta, s0, lengths, marks, y)

    def backward(self, q, k, v, g, beta, marks, dy, ds_end=None, lengths=None, stream=None):
        """dq, dk, dv, dg (None without a decay), dbeta and ds0, from the marks of a forward call on the same inputs."""
        if stream is not None:
            with _pool(stream):
                return self.backward(q, k, v, g, beta, marks, dy, ds_end, lengths)
        return self._ops.delta_backward(self._handle, q, k, v, g, beta, marks, dy, ds_end, lengths)

    def step(self, q, k, v, g, beta, state, new_state=None, active=None, y=None, stream=None):
        """One token: q, k [B, Hk * Dk], v [B, H * Dv], g, beta [B, H] -> y [B, H * Dv]; the states are replaced, or left and the new ones
        written to new_state."""
        if stream is not None:
            with _pool(stream):
                return self.step(q, k, v, g, beta, state, new_state, active, y)
        return self._ops.delta_step(self._handle, q, k, v, g, beta, state, new_state, active, y)


class Heads:
    """Queries [B, Hq * D, L_1..L_N] and keys [B, Hk * D, L_1..L_N] as heads: the norm over each head's channels ("rms", "l2" or "none") with
    weights g_q, g_k [D], then the pairs (i, i + D/2) turned by their position: the first axes[0] pairs on the first axis of the grid,
    the next axes[1] on the second and so on, the j-th of an axis at base^(-j / pairs); pairs behind them stay.  Positions are the
    grid's, or int32 [B, N, L_1..L_N].  Holds the shape only."""

    def __init__(self, dims, B: int, Hq: int, Hk: int, D: int, dtype=torch.float32, norm: str = "rms", axes=None, base: float = 10000.0, eps: float = 1e-6):
        self.dims = tuple(int(d) for d in dims)
        self.axes = (0,) * len(self.dims) if axes is None else tuple(int(n) for n in axes)
        self.B, self.Hq, self.Hk, self.D, self.dtype, self.norm, self.base, self.eps = int(B), int(Hq), int(Hk), int(D), dtype, norm, float(base), float(eps)
        code = {"none": HYENAND_NORM_NONE, "rms": HYENAND_NORM_RMS, "l2": HYENAND_NORM_L2}[norm]
        if len(self.axes) != len(self.dims):
            raise ValueError("axes must name a number of pairs for every axis of the grid")
        if min(self.axes, default=0) < 0 or 2 * sum(self.axes) > self.D:
            raise ValueError("the axes have more pairs than a head")
        work = hyenand_heads_workspace_bytes(len(self.dims), self.dims, self.B, self.Hq, self.Hk, self.D, _DTYPES[dtype])
        if work < 1:
            raise ValueError(hyenand_last_error())
        self._ops = _calls()
        self._handle = self._ops.make_heads(self.dims, self.axes, self.B, self.Hq, self.Hk, self.D, _DTYPES[dtype], code, self.base, self.eps, work,
                                            _address("hyenand_heads_forward"), _address("hyenand_heads_backward"), _check)

    def forward(self, q, k, g_q=None, g_k=None, positions=None, q_out=None, k_out=None, stream=None):
        """(q, k) normalised and turned; q_out may be q, k_out may be k."""
        if stream is not None:
            with _pool(stream):
                return self.forward(q, k, g_q, g_k, positions, q_out, k_out)
        return self._ops.heads_forward(self._handle, q, k, g_q, g_k, positions, q_out, k_out)

    def backward(self, q, k, dq_out, dk_out, g_q=None, g_k=None, positions=None, stream=None):
        """dq, dk, dg_q, dg_k (None for a weight that was not given), from the forward's inputs."""
        if stream is not None:
            with _pool(stream):
                return self.backward(q, k, dq_out, dk_out, g_q, g_k, positions)
        return self._ops.heads_backward(self._handle, q, k, dq_out, dk_out, g_q, g_k, positions)


class Block:
    """Between two mixers of a residual stream: r = x + scale * dropout(act(z) * RMSNorm(m, g_post)), n = RMSNorm(r, g_pre), the norms
    over the channels of each token of [B, C, L_1..L_N].  Weights that are not given leave their part out.  Holds the shape only."""

    def __init__(self, dims, B: int, C: int, dtype=torch.float32, gate: str = "none", eps: float = 1e-6, p: float = 0.0, site: int = 0):
        self.dims = tuple(int(d) for d in dims)
        self.B, self.C, self.dtype, self.gate, self.eps, self.p, self.site = int(B), int(C), dtype, gate, float(eps), float(p), int(site)
        code = {"none": HYENAND_GATE_NONE, "sigmoid": HYENAND_GATE_SIGMOID, "silu": HYENAND_GATE_SILU}[gate]
        T = math.prod(self.dims)
        if min((self.B, self.C) + self.dims) < 1:
            raise ValueError("B, C and every extent must be >= 1")
        self._ops = _calls()
        self._handle = self._ops.make_block(self.dims, self.B, self.C, T, _DTYPES[dtype], code, self.eps, self.p, self.site,
                                            hyenand_block_workspace_bytes(self.B, self.C, T, _DTYPES[dtype]), _address("hyenand_block_forward"),
                                            _address("hyenand_block_backward"), _check)

    def forward(self, x, m, z=None, g_post=None, scale=None, g_pre=None, rng=None, stats: bool = False, stream=None):
        """(r, n), n None without g_pre; with stats=True what `backward` needs of this call as a third."""
        if stream is not None:
            with _pool(stream):
                return self.forward(x, m, z, g_post, scale, g_pre, rng, stats)
        return self._ops.block_forward(self._handle, x, m, z, g_post, scale, g_pre, rng, stats)

    def backward(self, x, m, stats, z=None, g_post=None, scale=None, g_pre=None, rng=None, dr=None, dn=None, stream=None):
        """dx, dm, dz, dg_post, dscale, dg_pre (None for what was not given), from the stats of a forward call on the same inputs; dn is
        given exactly with g_pre, dr may be None (zero) beside it."""
        if stream is not None:
            with _pool(stream):
                return self.backward(x, m, stats, z, g_post, scale, g_pre, rng, dr, dn)
        return self._ops.block_backward(self._handle, x, m, stats, z, g_post, scale, g_pre, rng, dr, dn)


class Dropout:
    """y = x / (1 - p) or 0, the mask drawn from rng (int64 [2] on the device, 16-byte aligned: seed, step) and site; the backward pass
    is the same call on dy."""

    def __init__(self, p: float, site: int = 0):
        self.p, self.site, self._ops, self._call = float(p), int(site), _calls(), _address("hyenand_dropout")
        if not -1 << 31 <= self.site < 1 << 31:
            raise OverflowError("site must fit in 32 bits")     # (cut off, it would be another dropout's)

    def __call__(self, x, rng, y=None, stream=None):
        if stream is not None:
            with _pool(stream):
                return self(x, rng, y)
        return self._ops.dropout(self._call, _check, self.p, self.site, x, rng, y)
