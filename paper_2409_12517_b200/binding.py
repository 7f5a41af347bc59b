"""Python binding of libfp8mlp.so: same names as the C ABI, argument marshalling only.

Every function takes torch CUDA tensors (PyTorch is used for device memory and streams),
passes their device pointers and the current CUDA stream to the C entry point of the same
name, and raises Fp8MlpError on a non-zero status.  No step of the method runs in Python,
and there is no fallback: if the CUDA library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes as C
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libfp8mlp.so"

OK, ERR_ARG, ERR_SHAPE, ERR_ALIGN, ERR_CUDA, ERR_TIMEOUT, ERR_STATE, ERR_TOO_LARGE = 0, -1, -2, -3, -4, -5, -6, -7
STATIC_SCRATCH_BYTES = 4 * 1024 * 1024
E4M3, E5M2 = 0, 1
BF16, F32 = 0, 1
SMOOTH, SAVE_FOR_BWD, H_BF16, GU_FP8 = 1, 2, 4, 8
SCALE_GIVEN, SCALE_FROM_CURRENT_AMAX, SCALE_GIVEN_WEIGHTS_CAST, SCALE_GIVEN_X_CAST, SCALE_GIVEN_BOTH_CAST = 0, 1, 2, 3, 4
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
NORM_L2, NORM_INF = 0, 1
MAX_EXPERTS, MAX_TOP_K = 1024, 32
NORM_WORKSPACE_BYTES = 16384
RMS_SAME, RMS_E4M3, RMS_E4M3_ROWS = 0, 1, 2
MAX_NORM_WIDTH, RMS_PARTIALS = 16384, 592
MXFP4, NVFP4 = 0, 1
WS_XQ, WS_W12Q, WS_W3Q, WS_HQ, WS_GU, WS_DYQ, WS_DZQ, WS_HB, WS_W3B = range(9)

EXPORTS = [
    "fp8mlp_create", "fp8mlp_destroy", "fp8mlp_strerror", "fp8mlp_last_cuda_error", "fp8mlp_status",
    "fp8mlp_workspace", "fp8mlp_launch_count", "fp8mlp_quantize", "fp8mlp_update_scales",
    "fp8mlp_forward", "fp8mlp_backward", "fp8mlp_gemm_fp8", "fp8mlp_profile_enable", "fp8mlp_profile_read",
    "fp8mlp_forward_static", "fp8mlp_adam_step", "fp8mlp_scale_from_amax",
    "fp8mlp_merge_weights", "fp8mlp_forward_merged", "fp8mlp_gemm_bf16",
    "fp8mlp_selftest_wait_timeout", "fp8mlp_adam_step_cast", "fp8mlp_gemm_plan", "fp8mlp_code_stats",
    "fp8mlp_route", "fp8mlp_route_backward", "fp8mlp_route_update_bias", "fp8mlp_dispatch_plan", "fp8mlp_dispatch",
    "fp8mlp_combine", "fp8mlp_combine_backward", "fp8mlp_grad_norm", "fp8mlp_clip_grads", "fp8mlp_adam_step_scaled",
    "fp8mlp_rmsnorm", "fp8mlp_rmsnorm_backward", "fp8mlp_fp4_scale_bytes", "fp8mlp_quantize_fp4", "fp8mlp_dequantize_fp4",
    "fp8mlp_gemm_fp4",
]
PHASES = ["quant_x", "quant_w12", "quant_w3", "gemm1_swiglu", "gemm2_down", "quant_dy", "dgrad2_swiglu_bwd",
          "wgrad3", "dgrad1", "wgrad12", "misc"]


class Fp8MlpError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().fp8mlp_strerror(code).decode()
        detail = lib().fp8mlp_last_cuda_error().decode() if code == ERR_CUDA else ""
        super().__init__(f"{where}: {msg} ({code}){' — ' + detail if detail else ''}")


class _Scales(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("x", "w12", "w3", "dy", "dz", "h", "gu")]


class _Amax(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("x", "w1", "w2", "w3", "dy", "dz", "h", "gu")]


class _AdamTensor(C.Structure):
    _fields_ = [("w", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("n", C.c_int64),
                ("scale_m_in", C.c_void_p), ("scale_v_in", C.c_void_p), ("scale_m_out", C.c_void_p),
                ("scale_v_out", C.c_void_p), ("amax_m", C.c_void_p), ("amax_v", C.c_void_p)]


class _GemmPlan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("cta_pairs", "tile_rows", "tile_cols", "m_tiles", "n_tiles", "k_stages", "split_k",
                                       "stages_per_share", "band_along_n", "band_tiles", "staged_stores")] + [("work_items", C.c_int64)]


class _AdamCast(C.Structure):
    _fields_ = [("dst", C.c_void_p), ("cols", C.c_int64), ("ld_dst", C.c_int64), ("scale", C.c_void_p),
                ("row_div", C.c_void_p), ("amax", C.c_void_p)]


class Router(C.Structure):
    """How tokens choose their experts (fp8mlp_router; made by new_router)."""
    _fields_ = [(n, C.c_int32) for n in ("n_experts", "top_k", "score", "n_groups", "top_groups", "group_top",
                                         "renormalise")] + [("scale", C.c_float)]


class _GradTensor(C.Structure):
    _fields_ = [("g", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32)]


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_lib = None


def lib():
    """The loaded shared library (built by build.py); raises if it is not there."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2409_12517_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(str(LIB_PATH))
        L.fp8mlp_strerror.restype = C.c_char_p
        L.fp8mlp_strerror.argtypes = [C.c_int]
        L.fp8mlp_last_cuda_error.restype = C.c_char_p
        L.fp8mlp_launch_count.restype = C.c_int64
        L.fp8mlp_create.argtypes = [C.POINTER(C.c_void_p), C.c_int64, C.c_int64, C.c_int64, C.c_uint32]
        L.fp8mlp_destroy.argtypes = [C.c_void_p]
        L.fp8mlp_status.argtypes = [C.c_void_p, C.c_void_p]
        L.fp8mlp_workspace.argtypes = [C.c_void_p, C.c_int, C.POINTER(C.c_void_p), C.POINTER(C.c_int64)]
        L.fp8mlp_quantize.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int, C.c_int, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        L.fp8mlp_update_scales.argtypes = [C.c_void_p, C.POINTER(_Amax), C.POINTER(_Scales), C.c_void_p]
        L.fp8mlp_forward.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                     C.POINTER(_Scales), C.POINTER(_Amax), C.c_void_p, C.c_void_p]
        L.fp8mlp_backward.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.POINTER(_Scales), C.POINTER(_Amax),
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.fp8mlp_gemm_fp8.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_int,
                                      C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.fp8mlp_forward_static.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_uint32, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_int, C.POINTER(_Scales), C.POINTER(_Amax),
                                            C.c_void_p, C.c_void_p]
        L.fp8mlp_selftest_wait_timeout.argtypes = [C.c_void_p, C.c_int64, C.c_void_p]
        L.fp8mlp_gemm_bf16.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_int, C.c_void_p, C.c_int,
                                       C.c_void_p, C.c_void_p]
        L.fp8mlp_merge_weights.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                           C.POINTER(_Scales), C.POINTER(_Amax), C.c_void_p]
        L.fp8mlp_forward_merged.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.POINTER(_Scales),
                                            C.POINTER(_Amax), C.c_void_p, C.c_void_p]
        L.fp8mlp_adam_step.argtypes = [C.POINTER(_AdamTensor), C.c_int, C.c_float, C.c_float, C.c_float, C.c_float,
                                       C.c_float, C.c_int64, C.c_void_p]
        L.fp8mlp_adam_step_cast.argtypes = [C.POINTER(_AdamTensor), C.POINTER(_AdamCast), C.c_int, C.c_float, C.c_float,
                                            C.c_float, C.c_float, C.c_float, C.c_int64, C.c_void_p]
        L.fp8mlp_code_stats.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.fp8mlp_gemm_plan.argtypes = [C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_int, C.POINTER(_GemmPlan)]
        L.fp8mlp_scale_from_amax.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
        L.fp8mlp_profile_enable.argtypes = [C.c_void_p, C.c_int]
        L.fp8mlp_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        p, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
        L.fp8mlp_route.argtypes = [C.POINTER(Router), i64, p, i32, i64, p, p, p, p]
        L.fp8mlp_route_backward.argtypes = [C.POINTER(Router), i64, p, i32, i64, p, p, p, i64, p]
        L.fp8mlp_route_update_bias.argtypes = [i32, p, f32, p, p]
        L.fp8mlp_dispatch_plan.argtypes = [i64, i32, i32, p, p, p, p, p]
        L.fp8mlp_dispatch.argtypes = [i64, i32, i64, i32, p, i64, p, p, i64, p]
        L.fp8mlp_combine.argtypes = [i64, i32, i64, i32, p, i64, p, p, p, i64, p]
        L.fp8mlp_combine_backward.argtypes = [i64, i32, i64, i32, p, i64, p, i64, p, p, p, p, p]
        L.fp8mlp_grad_norm.argtypes = [C.POINTER(_GradTensor), i32, i32, f32, p, p, p]
        L.fp8mlp_clip_grads.argtypes = [C.POINTER(_GradTensor), i32, i32, f32, p, p, p]
        L.fp8mlp_adam_step_scaled.argtypes = [C.POINTER(_AdamTensor), C.POINTER(_AdamCast), i32, p, f32, f32, f32, f32,
                                              f32, i64, p]
        L.fp8mlp_rmsnorm.argtypes = [i64, i64, i32, p, i64, p, i64, p, i64, p, f32, i32, p, i64, p, p, p, p]
        L.fp8mlp_rmsnorm_backward.argtypes = [i64, i64, i32, p, i64, p, i64, p, p, p, i64, p, i64, p, p, p]
        L.fp8mlp_fp4_scale_bytes.restype = i64
        L.fp8mlp_fp4_scale_bytes.argtypes = [i32, i64, i64]
        L.fp8mlp_quantize_fp4.argtypes = [p, i32, i64, i64, i64, i32, i32, i32, p, p, p, i64, p, p]
        L.fp8mlp_dequantize_fp4.argtypes = [p, i64, p, p, i64, i64, i32, p, i32, i64, p]
        L.fp8mlp_gemm_fp4.argtypes = [i64, i64, i64, i32, p, i64, p, p, p, i64, p, p, p, i32, i64, p]
        missing = [name for name in EXPORTS if not hasattr(L, name)]
        if missing:
            raise RuntimeError(f"{LIB_PATH} does not export {missing}")
        _lib = L
    return _lib


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return C.c_void_p(t.data_ptr())


def _stream(here=None):
    """The current stream's handle (here: the current GPU, if the caller has asked for it).  torch.cuda.current_stream()
    builds a stream object around it, which takes longer (3.4 us) than a launch; the accessor that torch's own generated
    code uses takes 0.1 us."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device() if here is None else here)


def _here():
    """The current GPU, to whose stream a call goes; None where there is none, which no tensor lies on."""
    try:
        return _device()
    except (RuntimeError, AssertionError):
        return None


def _check(code: int, where: str):
    if code != OK:
        raise Fp8MlpError(code, where)


def _scales(s: dict) -> _Scales:
    return _Scales(*[(s[n].data_ptr() if s.get(n) is not None else None) for n in ("x", "w12", "w3", "dy", "dz", "h", "gu")])


def _amax(a: dict | None):
    if a is None:
        return None
    return _Amax(*[(a[n].data_ptr() if a.get(n) is not None else None) for n in ("x", "w1", "w2", "w3", "dy", "dz", "h", "gu")])


def fp8mlp_launch_count() -> int:
    return int(lib().fp8mlp_launch_count())


def fp8mlp_create(T_max: int, d_model: int, d_ff: int, flags: int) -> int:
    """Returns the context handle (an integer address)."""
    h = C.c_void_p()
    _check(lib().fp8mlp_create(C.byref(h), T_max, d_model, d_ff, flags), "fp8mlp_create")
    return h.value


def fp8mlp_destroy(ctx: int) -> None:
    _check(lib().fp8mlp_destroy(C.c_void_p(ctx)), "fp8mlp_destroy")


def fp8mlp_status(ctx: int | None) -> int:
    """Synchronises the current stream and returns OK or ERR_TIMEOUT (does not raise); ctx None: of the products without one."""
    return int(lib().fp8mlp_status(C.c_void_p(ctx), _stream()))


def fp8mlp_selftest_wait_timeout(ctx: int | None, timeout_us: int) -> None:
    """Runs a kernel whose bounded wait must time out; afterwards fp8mlp_status reports ERR_TIMEOUT once."""
    _check(lib().fp8mlp_selftest_wait_timeout(C.c_void_p(ctx), timeout_us, _stream()), "fp8mlp_selftest_wait_timeout")


class WorkspacePointer(int):
    """Address of a context's buffer that knows how many bytes there are from it on."""
    nbytes: int

    def __new__(cls, address: int, nbytes: int):
        p = super().__new__(cls, address)
        p.nbytes = nbytes
        return p

    def __add__(self, offset: int):
        """The address so many bytes on, as one that knows its size; outside the buffer, a plain number."""
        return WorkspacePointer(int(self) + offset, self.nbytes - offset) if 0 <= offset <= self.nbytes else int(self) + offset


def fp8mlp_workspace(ctx: int, which: int):
    """(device pointer, bytes) of one of the WS_* buffers; the pointer is a WorkspacePointer."""
    p, n = C.c_void_p(), C.c_int64()
    _check(lib().fp8mlp_workspace(C.c_void_p(ctx), which, C.byref(p), C.byref(n)), "fp8mlp_workspace")
    return WorkspacePointer(p.value or 0, n.value), n.value


def fp8mlp_profile_enable(ctx: int, on: bool) -> None:
    _check(lib().fp8mlp_profile_enable(C.c_void_p(ctx), int(on)), "fp8mlp_profile_enable")


def fp8mlp_profile_read(ctx: int) -> dict:
    """{phase name: (milliseconds, brackets)} accumulated since the last read."""
    n = len(PHASES)
    ms, cnt = (C.c_double * n)(), (C.c_int64 * n)()
    _check(lib().fp8mlp_profile_read(C.c_void_p(ctx), ms, cnt), "fp8mlp_profile_read")
    return {PHASES[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}


def fp8mlp_quantize(src, fp8_fmt: int, scale_mode: int, scale, amax, row_mul, dst, ld_dst: int | None = None) -> None:
    """src: 2-D bf16 or fp32 tensor; dst: uint8 tensor; scale/amax: 1-element fp32 tensors."""
    rows, cols = src.shape
    dtype = {torch.bfloat16: BF16, torch.float32: F32}[src.dtype]
    ld = cols if ld_dst is None else ld_dst
    _check(lib().fp8mlp_quantize(_ptr(src), dtype, rows, cols, fp8_fmt, scale_mode, _ptr(scale), _ptr(amax),
                                 _ptr(row_mul), _ptr(dst), ld, _stream()), "fp8mlp_quantize")


def fp8mlp_update_scales(ctx: int, amax: dict, scales: dict) -> None:
    a, s = _amax(amax), _scales(scales)
    _check(lib().fp8mlp_update_scales(C.c_void_p(ctx), C.byref(a), C.byref(s), _stream()), "fp8mlp_update_scales")


def fp8mlp_forward(ctx: int, T: int, x, W1, W2, W3, scale_mode: int, scales: dict, amax: dict | None, y) -> None:
    s, a = _scales(scales), _amax(amax)
    _check(lib().fp8mlp_forward(C.c_void_p(ctx), T, _ptr(x), _ptr(W1), _ptr(W2), _ptr(W3), scale_mode, C.byref(s),
                                C.byref(a) if a is not None else None, _ptr(y), _stream()), "fp8mlp_forward")


def fp8mlp_forward_static(T: int, d_model: int, d_ff: int, flags: int, x, W1, W2, W3, scale_mode: int,
                          scales: dict, amax: dict | None, y) -> None:
    """Forward for callers that cannot allocate device memory: no context, the library's built-in
    4 MiB scratch instead (shapes beyond it raise ERR_TOO_LARGE).  Calls that overlap on the GPU race."""
    s, a = _scales(scales), _amax(amax)
    _check(lib().fp8mlp_forward_static(T, d_model, d_ff, flags, _ptr(x), _ptr(W1), _ptr(W2), _ptr(W3), scale_mode,
                                       C.byref(s), C.byref(a) if a is not None else None, _ptr(y), _stream()),
           "fp8mlp_forward_static")


def fp8mlp_backward(ctx: int, T: int, dy, scale_mode: int, scales: dict, amax: dict | None, dx, dW1, dW2, dW3) -> None:
    s, a = _scales(scales), _amax(amax)
    _check(lib().fp8mlp_backward(C.c_void_p(ctx), T, _ptr(dy), scale_mode, C.byref(s),
                                 C.byref(a) if a is not None else None, _ptr(dx), _ptr(dW1), _ptr(dW2), _ptr(dW3),
                                 _stream()), "fp8mlp_backward")


def fp8mlp_gemm_fp8(M: int, N: int, K: int, A, a_kmajor: bool, a_fmt: int, B, b_kmajor: bool, b_fmt: int,
                    scale_a, scale_b, out) -> None:
    _check(lib().fp8mlp_gemm_fp8(M, N, K, _ptr(A), int(a_kmajor), a_fmt, _ptr(B), int(b_kmajor), b_fmt,
                                 _ptr(scale_a), _ptr(scale_b), _ptr(out), _stream()), "fp8mlp_gemm_fp8")


def fp8mlp_merge_weights(ctx: int, W1, W2, W3, s, scale_mode: int, scales: dict, amax: dict | None) -> None:
    sc, a = _scales(scales), _amax(amax)
    _check(lib().fp8mlp_merge_weights(C.c_void_p(ctx), _ptr(W1), _ptr(W2), _ptr(W3), _ptr(s), scale_mode, C.byref(sc),
                                      C.byref(a) if a is not None else None, _stream()), "fp8mlp_merge_weights")


def fp8mlp_forward_merged(ctx: int, T: int, x, scale_mode: int, scales: dict, amax: dict | None, y) -> None:
    sc, a = _scales(scales), _amax(amax)
    _check(lib().fp8mlp_forward_merged(C.c_void_p(ctx), T, _ptr(x), scale_mode, C.byref(sc),
                                       C.byref(a) if a is not None else None, _ptr(y), _stream()), "fp8mlp_forward_merged")


def _adam_tensors(tensors: list):
    arr = (_AdamTensor * len(tensors))()
    for a, t in zip(arr, tensors):
        a.w, a.g, a.m, a.v, a.n = t["w"].data_ptr(), t["g"].data_ptr(), t["m"].data_ptr(), t["v"].data_ptr(), t["w"].numel()
        for k in ("scale_m_in", "scale_v_in", "scale_m_out", "scale_v_out", "amax_m", "amax_v"):
            setattr(a, k, t[k].data_ptr())
    return arr


def _adam_casts(casts: list, count: int):
    carr = (_AdamCast * count)()
    for c, d in zip(carr, casts):
        if d is None:
            continue
        c.dst = d["dst"] if isinstance(d["dst"], int) else d["dst"].data_ptr()
        c.cols, c.ld_dst, c.scale = d["cols"], d["ld_dst"], d["scale"].data_ptr()
        c.row_div = d["row_div"].data_ptr() if d.get("row_div") is not None else None
        c.amax = d["amax"].data_ptr() if d.get("amax") is not None else None
    return carr


def fp8mlp_adam_step(tensors: list, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float,
                     step: int) -> None:
    """tensors: dicts with torch tensors w, g (fp32), m, v (uint8 codes) and 1-element fp32 tensors
    scale_m_in, scale_v_in, scale_m_out, scale_v_out, amax_m, amax_v.  Everything is updated in place."""
    _check(lib().fp8mlp_adam_step(_adam_tensors(tensors), len(tensors), lr, beta1, beta2, eps, weight_decay, step,
                                  _stream()), "fp8mlp_adam_step")


def fp8mlp_adam_step_cast(tensors: list, casts: list, lr: float, beta1: float, beta2: float, eps: float,
                          weight_decay: float, step: int) -> None:
    """fp8mlp_adam_step that also writes the E4M3 codes of the updated weights.  casts: one entry per tensor, None or a
    dict with dst (device pointer as int, or a uint8 tensor), cols, ld_dst, scale (1-element fp32 tensor), and
    optionally row_div (fp32 tensor, one per row) and amax (1-element fp32 tensor)."""
    _check(lib().fp8mlp_adam_step_cast(_adam_tensors(tensors), _adam_casts(casts, len(tensors)), len(tensors), lr, beta1,
                                       beta2, eps, weight_decay, step, _stream()), "fp8mlp_adam_step_cast")


def fp8mlp_adam_step_scaled(tensors: list, casts: list | None, grad_scale, lr: float, beta1: float, beta2: float,
                            eps: float, weight_decay: float, step: int) -> None:
    """The same two steps (casts None: without the codes) on the gradients times grad_scale, a 1-element fp32 CUDA tensor,
    e.g. norm_coef[1:] of fp8mlp_grad_norm."""
    here = _here()
    _check(lib().fp8mlp_adam_step_scaled(_adam_tensors(tensors), None if casts is None else _adam_casts(casts, len(tensors)),
                                         len(tensors), _as(grad_scale, _F32, 1, "grad_scale", here), lr, beta1, beta2, eps,
                                         weight_decay, step, _stream(here)), "fp8mlp_adam_step_scaled")


def fp8mlp_code_stats(codes, fp8_fmt: int, counts, ld: int | None = None) -> None:
    """codes: 2-D uint8 CUDA tensor (row stride ld, default cols); counts: int64 CUDA tensor of 2 elements, receives
    (zero codes, codes at the largest finite magnitude)."""
    rows, cols = codes.shape
    _check(lib().fp8mlp_code_stats(_ptr(codes), rows, cols, cols if ld is None else ld, fp8_fmt, C.c_void_p(counts.data_ptr()),
                                   C.c_void_p(counts.data_ptr() + 8), _stream()), "fp8mlp_code_stats")


GEMM_F32_OUT, GEMM_BF16_OUT, GEMM_SWIGLU_FWD, GEMM_SWIGLU_BWD = 0, 1, 2, 3


def fp8mlp_gemm_plan(kind: int, M: int, N: int, K: int, sm_count: int = 148, with_workspace: bool = True) -> dict:
    """How the library would tile and schedule one GEMM (host arithmetic only; works without a GPU)."""
    p = _GemmPlan()
    _check(lib().fp8mlp_gemm_plan(kind, M, N, K, sm_count, int(with_workspace), C.byref(p)), "fp8mlp_gemm_plan")
    return {n: getattr(p, n) for n, _ in _GemmPlan._fields_}


def fp8mlp_scale_from_amax(amax, fp8_fmt: int, scale) -> None:
    _check(lib().fp8mlp_scale_from_amax(_ptr(amax), fp8_fmt, _ptr(scale), _stream()), "fp8mlp_scale_from_amax")


def fp8mlp_gemm_bf16(M: int, N: int, K: int, A, a_kmajor: bool, B, b_kmajor: bool, out) -> None:
    _check(lib().fp8mlp_gemm_bf16(M, N, K, _ptr(A), int(a_kmajor), _ptr(B), int(b_kmajor), _ptr(out), _stream()),
           "fp8mlp_gemm_bf16")


# ---------------------------------------------------------------- experts of one layer, and clipping

_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}
_F32, _I32, _U8 = torch.float32, torch.int32, torch.uint8


def _as(t, dtype, numel, what, here):
    """Device pointer of a contiguous tensor of the given type and size on the current GPU."""
    if t.dtype is not dtype or t.numel() != numel or t.get_device() != here or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous CUDA tensor of {numel} {dtype} elements on the current GPU is needed, "
                         f"got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _matrix(t, cols, what, here, dtype=None):
    """(rows, pointer, type, row stride) of a 2-D tensor on the current GPU whose rows are contiguous; any row stride >= its
    columns."""
    shape, code = t.shape, _DTYPES.get(t.dtype)
    if len(shape) != 2 or shape[1] != cols or code is None or (dtype is not None and t.dtype is not dtype) or t.get_device() != here:
        raise ValueError(f"{what}: a 2-D CUDA tensor of {cols} columns in {dtype or 'bfloat16 or float32'} on the current GPU is "
                         f"needed, got {tuple(shape)} {t.dtype} on {t.device}")
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{what}: the elements of a row must be neighbours")
    return shape[0], t.data_ptr(), code, ld if ld >= cols or shape[0] > 1 else cols      # a single row's stride may be anything


def new_router(n_experts: int, top_k: int, score: int = SCORE_SOFTMAX, n_groups: int = 1, top_groups: int = 1,
               group_top: int = 1, renormalise: bool = True, scale: float = 1.0) -> Router:
    return Router(n_experts, top_k, score, n_groups, top_groups, group_top, int(renormalise), scale)


def fp8mlp_route(router: Router, logits, bias, experts, weights) -> None:
    """logits: [T, n_experts] bf16 or fp32, any row stride; bias: fp32 [n_experts] or None; receives experts (int32
    [T, top_k]) and weights (fp32 [T, top_k])."""
    E, here = router.n_experts, _here()
    T, ptr, dtype, ld = _matrix(logits, E, "logits", here)
    n = T * router.top_k
    _check(lib().fp8mlp_route(router, T, ptr, dtype, ld, None if bias is None else _as(bias, _F32, E, "bias", here),
                              _as(experts, _I32, n, "experts", here), _as(weights, _F32, n, "weights", here), _stream(here)),
           "fp8mlp_route")


def fp8mlp_route_backward(router: Router, logits, experts, d_weights, d_logits) -> None:
    """d_logits (type of the logits, any row stride) from d_weights (fp32 [T, top_k]) for the experts the forward chose."""
    E, here = router.n_experts, _here()
    T, ptr, dtype, ld = _matrix(logits, E, "logits", here)
    d_rows, d_ptr, _, ld_d = _matrix(d_logits, E, "d_logits", here, logits.dtype)
    n = T * router.top_k
    if d_rows != T:
        raise ValueError("d_logits: not as many rows as logits")
    _check(lib().fp8mlp_route_backward(router, T, ptr, dtype, ld, _as(experts, _I32, n, "experts", here),
                                       _as(d_weights, _F32, n, "d_weights", here), d_ptr, ld_d, _stream(here)),
           "fp8mlp_route_backward")


def fp8mlp_route_update_bias(counts, rate: float, bias) -> None:
    """bias (fp32 [n_experts], in place) moves by rate towards the experts with fewer rows than the mean (counts, int32)."""
    n, here = bias.numel(), _here()
    _check(lib().fp8mlp_route_update_bias(n, _as(counts, _I32, n, "counts", here), rate, _as(bias, _F32, n, "bias", here),
                                          _stream(here)), "fp8mlp_route_update_bias")


def fp8mlp_dispatch_plan(experts, n_experts: int, counts, offsets, rows) -> None:
    """experts: int32 [T, top_k]; receives counts (int32 [n_experts]), offsets (int32 [n_experts + 1]) and rows (int32
    [T, top_k])."""
    (T, k), here = experts.shape, _here()
    _check(lib().fp8mlp_dispatch_plan(T, k, n_experts, _as(experts, _I32, T * k, "experts", here),
                                      _as(counts, _I32, n_experts, "counts", here),
                                      _as(offsets, _I32, n_experts + 1, "offsets", here),
                                      _as(rows, _I32, T * k, "rows", here), _stream(here)), "fp8mlp_dispatch_plan")


def _rows_pair(token, expert, rows, token_name, expert_name):
    """What dispatch and combine pass alike: (current GPU, tokens, slots, d, type, token pointer and row stride, expert pointer and
    rows, rows pointer)."""
    T, k = rows.shape
    n, d = expert.shape
    here = _here()
    have, ptr, dtype, ld = _matrix(token, d, token_name, here, expert.dtype)
    if have != T:
        raise ValueError(f"{token_name}: {have} rows, but rows speaks of {T} tokens")
    return here, T, k, d, dtype, ptr, ld, _as(expert, expert.dtype, n * d, expert_name, here), n, _as(rows, _I32, T * k, "rows", here)


def fp8mlp_dispatch(x, rows, xe) -> None:
    """xe[rows[t, j]] = x[t]; x: [T, d] bf16 or fp32, any row stride; xe: [n, d] of the same type, contiguous."""
    here, T, k, d, dtype, ptr, ld, xe_ptr, n, rows_ptr = _rows_pair(x, xe, rows, "x", "xe")
    _check(lib().fp8mlp_dispatch(T, k, d, dtype, ptr, ld, rows_ptr, xe_ptr, n, _stream(here)), "fp8mlp_dispatch")


def fp8mlp_combine(ye, rows, weights, y) -> None:
    """y[t] = sum_j weights[t, j] ye[rows[t, j]]; weights fp32 [T, top_k] or None (= 1); y: [T, d], any row stride."""
    here, T, k, d, dtype, ptr, ld, ye_ptr, n, rows_ptr = _rows_pair(y, ye, rows, "y", "ye")
    _check(lib().fp8mlp_combine(T, k, d, dtype, ye_ptr, n, rows_ptr,
                                None if weights is None else _as(weights, _F32, T * k, "weights", here), ptr, ld, _stream(here)),
           "fp8mlp_combine")


def fp8mlp_combine_backward(dy, ye, rows, weights, dye, d_weights) -> None:
    """dye[rows[t, j]] = weights[t, j] dy[t] and d_weights[t, j] = <dy[t], ye[rows[t, j]]> (fp32 [T, top_k])."""
    here, T, k, d, dtype, ptr, ld, ye_ptr, n, rows_ptr = _rows_pair(dy, ye, rows, "dy", "ye")
    _check(lib().fp8mlp_combine_backward(T, k, d, dtype, ptr, ld, ye_ptr, n, rows_ptr,
                                         _as(weights, _F32, T * k, "weights", here), _as(dye, ye.dtype, n * d, "dye", here),
                                         _as(d_weights, _F32, T * k, "d_weights", here), _stream(here)),
           "fp8mlp_combine_backward")


class GradList:
    """The tensors of one clipping call, marshalled once; a program whose gradients stay where they are keeps it (it
    holds the tensors, and addresses only - every call reads the gradients anew)."""

    def __init__(self, grads, outs):
        self.tensors = (list(grads), list(grads if outs is None else outs))
        if len(self.tensors[0]) != len(self.tensors[1]):
            raise ValueError("as many outputs as gradients are needed")
        self.count = len(self.tensors[0])
        self.array = (_GradTensor * max(self.count, 1))()
        self.device = _here()
        for a, g, o in zip(self.array, *self.tensors):
            if g.dtype not in _DTYPES:
                raise ValueError(f"gradients are bfloat16 or float32, not {g.dtype}")
            a.g, a.out, a.n, a.dtype = (_as(g, g.dtype, g.numel(), "gradient", self.device),
                                        _as(o, g.dtype, g.numel(), "output", self.device), g.numel(), _DTYPES[g.dtype])


def new_grad_list(grads, outs=None) -> GradList:
    """grads: contiguous bf16 / fp32 CUDA tensors; outs: where the clipped ones go (default: in place)."""
    return GradList(grads, outs)


def new_norm_workspace(device="cuda"):
    return torch.empty(NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=device)


def _clip_args(grads, norm_kind, max_norm, norm_coef, workspace):
    here = _here()
    if grads.device != here:
        raise ValueError(f"gradients: the list was made for GPU {grads.device}, the current one is {here}")
    return (grads.array, grads.count, norm_kind, max_norm, _as(norm_coef, _F32, 2, "norm_coef", here),
            _as(workspace, _U8, NORM_WORKSPACE_BYTES, "workspace", here), _stream(here))


def fp8mlp_grad_norm(grads: GradList, norm_kind: int, max_norm: float, norm_coef, workspace) -> None:
    """norm_coef (fp32 [2]) receives the global norm and min(1, max_norm / (norm + 1e-6))."""
    _check(lib().fp8mlp_grad_norm(*_clip_args(grads, norm_kind, max_norm, norm_coef, workspace)), "fp8mlp_grad_norm")


def fp8mlp_clip_grads(grads: GradList, norm_kind: int, max_norm: float, norm_coef, workspace) -> None:
    """fp8mlp_grad_norm, and out = g * coefficient for every tensor of the list."""
    _check(lib().fp8mlp_clip_grads(*_clip_args(grads, norm_kind, max_norm, norm_coef, workspace)), "fp8mlp_clip_grads")


# ---------------------------------------------------------------- the norm in front of the block

def _rows_like(t, shape, dtype, what, here):
    """(pointer, row stride) of a tensor of one shape [rows, cols] and type whose rows are contiguous, or (None, 0)."""
    if t is None:
        return None, 0
    if t.dtype is dtype and t.shape == shape and t.get_device() == here and t.is_contiguous():      # the usual case, quickly
        return t.data_ptr(), shape[1]
    have, ptr, _, ld = _matrix(t, shape[1], what, here, dtype)
    if have != shape[0]:
        raise ValueError(f"{what}: {have} rows, {shape[0]} are needed")
    return ptr, ld


def _floats(t, numel, what, here):
    """Device pointer of a contiguous fp32 tensor of that size on the current GPU, or None."""
    if t is None:
        return None
    if t.dtype is not _F32 or t.numel() != numel or t.get_device() != here or not t.is_contiguous():
        _as(t, _F32, numel, what, here)
    return t.data_ptr()


def fp8mlp_rmsnorm(x, residual, gain, eps: float, y, h=None, out: int = RMS_SAME, scale=None, amax=None, rstd=None) -> None:
    """h = x + residual, y = h / rms(h) * gain.  x, residual, h: [T, d] bf16 or fp32, any row stride; residual, gain (fp32
    [d]), h, amax (1-element fp32) and rstd (fp32 [T]) may be None; h may be x or residual, in the same rows.  y by `out`: RMS_SAME: [T, d] of
    x's type; RMS_E4M3: codes (uint8 [T, d], or a context's buffer by its WorkspacePointer, WS_XQ with rows of d bytes) of
    y * scale (1-element fp32, read); RMS_E4M3_ROWS: codes, scale (fp32 [T]) is written."""
    here = _here()
    shape, dtype = x.shape, x.dtype
    if len(shape) != 2 or dtype not in _DTYPES:
        raise ValueError(f"x: a 2-D bfloat16 or float32 tensor is needed, got {tuple(shape)} {dtype}")
    T, d = shape
    # (the usual case is tested in place: eight tensors, and a call into a helper for each would be a tenth of a small norm's time)
    if x.is_contiguous() and x.get_device() == here:
        x_ptr, ld_x = x.data_ptr(), d
    else:
        x_ptr, ld_x = _rows_like(x, shape, dtype, "x", here)
    if residual is None:
        r_ptr, ld_r = None, 0
    elif residual.dtype is dtype and residual.shape == shape and residual.is_contiguous() and residual.get_device() == here:
        r_ptr, ld_r = residual.data_ptr(), d
    else:
        r_ptr, ld_r = _rows_like(residual, shape, dtype, "residual", here)
    if h is None:
        h_ptr, ld_h = None, 0
    elif h.dtype is dtype and h.shape == shape and h.is_contiguous() and h.get_device() == here:
        h_ptr, ld_h = h.data_ptr(), d
    else:
        h_ptr, ld_h = _rows_like(h, shape, dtype, "h", here)
    if isinstance(y, int):
        if out == RMS_SAME or not isinstance(y, WorkspacePointer) or T * d > y.nbytes:
            raise ValueError(f"y: {T * d} bytes of codes go to a uint8 tensor or to a context's buffer of that size (the pointer from "
                             f"fp8mlp_workspace), got {f'{y.nbytes} bytes' if isinstance(y, WorkspacePointer) else 'a bare address'}")
        y_ptr, ld_y = y, d
    elif out == RMS_SAME:
        y_ptr, ld_y = _rows_like(y, shape, dtype, "y", here)
    elif y.dtype is _U8 and y.shape == shape and y.is_contiguous() and y.get_device() == here:
        y_ptr, ld_y = y.data_ptr(), d
    else:
        y_ptr, ld_y = _bytes(y, T, d, "y", here)
    _check(lib().fp8mlp_rmsnorm(T, d, _DTYPES[dtype], x_ptr, ld_x, r_ptr, ld_r, h_ptr, ld_h, _floats(gain, d, "gain", here), eps, out,
                                y_ptr, ld_y, _floats(scale, T if out == RMS_E4M3_ROWS else 1, "scale", here),
                                _floats(amax, 1, "amax", here), _floats(rstd, T, "rstd", here), _stream(here)), "fp8mlp_rmsnorm")


def fp8mlp_rmsnorm_backward(dy, h, gain, rstd, dh, dx, d_gain, workspace) -> None:
    """dx [T, d] (may be dy or dh, in the same rows) and d_gain (fp32 [d], or None) from dy, the stored h and rstd; dh: what reached h along the
    residual stream, or None; workspace: new_rmsnorm_workspace(d), or None without d_gain."""
    here = _here()
    shape, dtype = h.shape, h.dtype
    if len(shape) != 2 or dtype not in _DTYPES:
        raise ValueError(f"h: a 2-D bfloat16 or float32 tensor is needed, got {tuple(shape)} {dtype}")
    T, d = shape
    if h.is_contiguous() and h.get_device() == here:
        h_ptr, ld_h = h.data_ptr(), d
    else:
        h_ptr, ld_h = _rows_like(h, shape, dtype, "h", here)
    if dy.dtype is dtype and dy.shape == shape and dy.is_contiguous() and dy.get_device() == here:
        dy_ptr, ld_dy = dy.data_ptr(), d
    else:
        dy_ptr, ld_dy = _rows_like(dy, shape, dtype, "dy", here)
    if dh is None:
        dh_ptr, ld_dh = None, 0
    elif dh.dtype is dtype and dh.shape == shape and dh.is_contiguous() and dh.get_device() == here:
        dh_ptr, ld_dh = dh.data_ptr(), d
    else:
        dh_ptr, ld_dh = _rows_like(dh, shape, dtype, "dh", here)
    if dx.dtype is dtype and dx.shape == shape and dx.is_contiguous() and dx.get_device() == here:
        dx_ptr, ld_dx = dx.data_ptr(), d
    else:
        dx_ptr, ld_dx = _rows_like(dx, shape, dtype, "dx", here)
    _check(lib().fp8mlp_rmsnorm_backward(T, d, _DTYPES[dtype], dy_ptr, ld_dy, h_ptr, ld_h, _floats(gain, d, "gain", here),
                                         _as(rstd, _F32, T, "rstd", here), dh_ptr, ld_dh, dx_ptr, ld_dx,
                                         _floats(d_gain, d, "d_gain", here), _floats(workspace, RMS_PARTIALS * d, "workspace", here),
                                         _stream(here)), "fp8mlp_rmsnorm_backward")


def new_rmsnorm_workspace(d: int, device="cuda"):
    return torch.empty(RMS_PARTIALS * d, dtype=torch.float32, device=device)


# ---------------------------------------------------------------- 4-bit operands

def _bytes(t, rows, cols, what, here):
    """(pointer, row stride) of a uint8 matrix whose rows are contiguous, at least `cols` long."""
    shape, strides = t.shape, t.stride()
    if len(shape) != 2 or t.dtype is not _U8 or shape[0] != rows or shape[1] < cols or t.get_device() != here or strides[1] != 1:
        raise ValueError(f"{what}: a 2-D uint8 CUDA tensor of {rows} rows of {cols} bytes on the current GPU is needed, got "
                         f"{tuple(shape)} {t.dtype} on {t.device}")
    return t.data_ptr(), strides[0] if rows > 1 else max(strides[0], shape[1])


class Fp4Operand:
    """A [rows, cols] matrix in 4 bits, its columns the contraction of a product: codes (uint8 [rows, at least cols / 2 rounded
    up to 16], a row stride that is a multiple of 16), block scales (uint8, fp8mlp_fp4_scale_bytes) and, for NVFP4, the tensor's scale (1-element fp32,
    None = 1).  Marshalled once: it holds the tensors and their addresses; what is in them is read anew by every call."""

    def __init__(self, fmt: int, rows: int, cols: int, codes, scales, scale=None, amax=None):
        self.fmt, self.rows, self.cols, self.device = fmt, rows, cols, codes.get_device()
        self._tensors = (codes, scales, scale, amax)
        self.codes_ptr, self.ld_codes = _bytes(codes, rows, (cols + 31) // 32 * 16, "codes", self.device)
        self.scales_ptr = _as(scales, _U8, fp8mlp_fp4_scale_bytes(fmt, rows, cols), "block scales", self.device)
        self.scale_ptr = None if scale is None else _as(scale, _F32, 1, "scale", self.device)
        self.amax_ptr = None if amax is None else _as(amax, _F32, 1, "amax", self.device)

    codes = property(lambda self: self._tensors[0])
    scales = property(lambda self: self._tensors[1])
    scale = property(lambda self: self._tensors[2])
    amax = property(lambda self: self._tensors[3])


def _operand(op, what, here):
    if op.device != here or here is None:
        raise ValueError(f"{what}: an operand on the current GPU is needed, this one is on {op.codes.device}")
    return op


def fp8mlp_fp4_scale_bytes(fmt: int, rows: int, cols: int) -> int:
    return int(lib().fp8mlp_fp4_scale_bytes(fmt, rows, cols))


def new_fp4(fmt: int, rows: int, cols: int, scale=None, device="cuda") -> Fp4Operand:
    """Buffers for a [rows, cols] operand; NVFP4: with the given tensor scale, or one of its own, initialised to 1."""
    if fmt == NVFP4 and scale is None:
        scale = torch.ones(1, dtype=torch.float32, device=device)
    return Fp4Operand(fmt, rows, cols, torch.empty((rows, (cols + 31) // 32 * 16), dtype=torch.uint8, device=device),
                      torch.empty(fp8mlp_fp4_scale_bytes(fmt, rows, cols), dtype=torch.uint8, device=device), scale,
                      torch.zeros(1, dtype=torch.float32, device=device))


def fp8mlp_quantize_fp4(src, operand: Fp4Operand, transpose: bool = False, scale_mode: int = SCALE_GIVEN, amax=None) -> None:
    """src: 2-D bf16 or fp32, any row stride; fills operand (of src, or of its transpose).  SCALE_FROM_CURRENT_AMAX (NVFP4)
    writes operand.scale first; amax (1-element fp32): receives max |src| (in that mode the operand's own if None)."""
    here = _here()
    shape, dtype = src.shape, src.dtype
    if shape != ((operand.cols, operand.rows) if transpose else (operand.rows, operand.cols)):
        raise ValueError(f"operand: {operand.rows} x {operand.cols}, but src is {tuple(shape)}{' (to be transposed)' if transpose else ''}")
    if dtype not in _DTYPES:
        raise ValueError(f"src: bfloat16 or float32 is needed, not {dtype}")
    ptr, ld = _rows_like(src, shape, dtype, "src", here)
    o = _operand(operand, "operand", here)
    amax_ptr = _as(amax, _F32, 1, "amax", here) if amax is not None else o.amax_ptr if scale_mode == SCALE_FROM_CURRENT_AMAX else None
    _check(lib().fp8mlp_quantize_fp4(ptr, _DTYPES[dtype], shape[0], shape[1], ld, 1 if transpose else 0, o.fmt, scale_mode, o.scale_ptr,
                                     amax_ptr, o.codes_ptr, o.ld_codes, o.scales_ptr, _stream(here)), "fp8mlp_quantize_fp4")


def fp8mlp_dequantize_fp4(operand: Fp4Operand, out) -> None:
    """out: [rows, cols] bf16 or fp32, any row stride, receives the values that the operand stands for."""
    here = _here()
    dtype = out.dtype
    if dtype not in _DTYPES:
        raise ValueError(f"out: bfloat16 or float32 is needed, not {dtype}")
    ptr, ld = _rows_like(out, (operand.rows, operand.cols), dtype, "out", here)
    o = _operand(operand, "operand", here)
    _check(lib().fp8mlp_dequantize_fp4(o.codes_ptr, o.ld_codes, o.scales_ptr, o.scale_ptr, o.rows, o.cols, o.fmt, ptr, _DTYPES[dtype], ld,
                                       _stream(here)), "fp8mlp_dequantize_fp4")


def fp8mlp_gemm_fp4(a: Fp4Operand, b: Fp4Operand, out) -> None:
    """out[m, n] = sum_k a[m, k] b[n, k]; out: [a.rows, b.rows] bf16 or fp32, any row stride."""
    here = _here()
    if a.fmt != b.fmt or a.cols != b.cols:
        raise ValueError(f"operands: formats {a.fmt} and {b.fmt}, contractions {a.cols} and {b.cols}")
    dtype = out.dtype
    if dtype not in _DTYPES:
        raise ValueError(f"out: bfloat16 or float32 is needed, not {dtype}")
    _operand(a, "a", here), _operand(b, "b", here)
    ptr, ld = _rows_like(out, (a.rows, b.rows), dtype, "out", here)
    _check(lib().fp8mlp_gemm_fp4(a.rows, b.rows, a.cols, a.fmt, a.codes_ptr, a.ld_codes, a.scales_ptr, a.scale_ptr, b.codes_ptr,
                                 b.ld_codes, b.scales_ptr, b.scale_ptr, ptr, _DTYPES[dtype], ld, _stream(here)), "fp8mlp_gemm_fp4")


# ---------------------------------------------------------------- conveniences (allocation only)

def new_scales(d_ff: int, device="cuda") -> dict:
    """Caller-owned scale buffers, initialised to 1."""
    s = {n: torch.ones(1, dtype=torch.float32, device=device) for n in ("x", "w12", "w3", "dy", "dz", "gu")}
    s["h"] = torch.ones(d_ff, dtype=torch.float32, device=device)
    return s


def new_amax(d_ff: int, device="cuda") -> dict:
    a = {n: torch.zeros(1, dtype=torch.float32, device=device) for n in ("x", "w1", "w2", "w3", "dy", "dz", "gu")}
    a["h"] = torch.zeros(d_ff, dtype=torch.float32, device=device)
    return a


class _DeviceBytes:
    """Exposes a raw device pointer through the CUDA array interface (zero-copy view for torch)."""

    def __init__(self, ptr: int, nbytes: int):
        self.__cuda_array_interface__ = {"shape": (nbytes,), "typestr": "|u1", "data": (ptr, False), "version": 2}


def workspace_tensor(ctx: int, which: int, shape, dtype):
    """A copy of the first prod(shape) elements of a workspace buffer, as a torch tensor (for tests)."""
    ptr, nbytes = fp8mlp_workspace(ctx, which)
    n = 1
    for s in shape:
        n *= s
    need = n * torch.empty(0, dtype=dtype).element_size()
    assert need <= nbytes
    if need == 0:
        return torch.empty(shape, dtype=dtype, device="cuda")
    raw = torch.as_tensor(_DeviceBytes(ptr, nbytes), device="cuda")
    return raw[:need].view(dtype).view(shape).clone()


def workspace_fill(ctx: int, which: int, byte: int) -> None:
    """Sets every byte of a workspace buffer (for tests: a poison pattern shows what a call failed to write)."""
    ptr, nbytes = fp8mlp_workspace(ctx, which)
    if nbytes:
        torch.as_tensor(_DeviceBytes(ptr, nbytes), device="cuda").fill_(byte)
