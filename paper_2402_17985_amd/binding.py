"""Thin Python binding of libfq.so (include/fq.h).

Argument marshalling only: every step of the path runs in the HIP kernels behind the C ABI.
PyTorch tensors are used as device buffers (`data_ptr()`) and for the current stream; nothing is
computed in PyTorch.  There is no fallback: if libfq.so is missing, loading raises.
"""
import ctypes
import os
from typing import Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfq.so")

FQ_F32, FQ_F16, FQ_BF16, FQ_I32 = 0, 1, 2, 3
FQ_OK = 0
ERR_NAMES = {1: "FQ_ERR_NULL", 2: "FQ_ERR_SHAPE", 3: "FQ_ERR_DTYPE", 4: "FQ_ERR_RANGE", 5: "FQ_ERR_ALIGN",
             6: "FQ_ERR_HIP", 7: "FQ_ERR_WORKSPACE"}

# every entry point include/fq.h declares
SYMBOLS = ["fq_last_error_string", "fq_version", "fq_flatten_plan", "fq_flatten_weights",
           "fq_weights_workspace_bytes", "fq_flatten_quant_act", "fq_act_workspace_bytes", "fq_gemm_i8",
           "fq_gemm_i4", "fq_linear", "fq_linear_workspace_bytes", "fq_gemm_bf16", "fq_gemm_select",
           "fq_threshold_boxplot", "fq_smooth_scales", "fq_channel_absmax", "fq_bmm_i8", "fq_bmm_i4",
           "fq_flatten_plan_xw", "fq_flatten_weights_split", "fq_flatten_quant_act_peel",
           "fq_gemm_i8_bias", "fq_gemm_i4_bias", "fq_linear_bias", "fq_linear_fused_a_i8", "fq_gemm_i4_e3m2",
           "fq_flatten_quant_act_noalloc", "fq_noalloc_scratch_bytes",
           "fq_kv_append", "fq_attn_cache_workspace_bytes", "fq_attn_cache", "fq_attn_prompt",
           # include/fq_peak.h: measurement hooks
           "fq_peak_mfma", "fq_peak_copy", "fq_peak_gemm_ticks", "fq_peak_wall_clock_khz"]
FQ_PEAK_I8, FQ_PEAK_BF16, FQ_PEAK_E3M2, FQ_PEAK_I8_NIBBLES = 0, 1, 2, 3
FQ_BITS_I4_E3M2 = 6   # the 4-bit quantizer with its values stored as 6-bit E3M2 codes


class FqError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERR_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Load libfq.so (built in-tree by paper_2402_17985_amd/build.py).  Raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} not found: build it with `python -m paper_2402_17985_amd.build` "
                                "(there is no CPU or PyTorch fallback)")
    L = ctypes.CDLL(LIB_PATH)
    c_int, c_float, c_size_t, vp = ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p
    L.fq_last_error_string.restype = ctypes.c_char_p
    L.fq_last_error_string.argtypes = []
    L.fq_version.restype = c_int
    L.fq_gemm_select.argtypes = [c_int]
    L.fq_flatten_plan.argtypes = [vp, c_int, c_float, c_int, vp, vp, c_int, ctypes.POINTER(c_int),
                                  ctypes.POINTER(c_int)]
    L.fq_threshold_boxplot.argtypes = [vp, c_int, c_float, ctypes.POINTER(c_float)]
    L.fq_smooth_scales.argtypes = [vp, vp, c_int, c_float, vp]
    L.fq_flatten_plan_xw.argtypes = [vp, c_float, vp, c_float, c_int, c_int, vp, vp, vp, vp, c_int,
                                     ctypes.POINTER(c_int), ctypes.POINTER(c_int)]
    L.fq_flatten_weights_split.argtypes = [vp, c_int, c_int, c_int, c_int, vp, vp, c_int, c_int, vp, vp, vp, c_size_t, vp]
    L.fq_flatten_quant_act_peel.argtypes = [vp, c_int, c_int, c_int, c_int, vp, vp, c_int, c_int, c_float, vp, vp, vp,
                                            vp, c_size_t, vp]
    L.fq_channel_absmax.argtypes = [vp, c_int, c_int, c_int, c_int, c_int, vp, vp]
    L.fq_flatten_weights.argtypes = [vp, c_int, c_int, c_int, c_int, vp, c_int, c_int, vp, vp, vp, c_size_t, vp]
    L.fq_weights_workspace_bytes.restype = c_size_t
    L.fq_weights_workspace_bytes.argtypes = [c_int, c_int]
    L.fq_flatten_quant_act.argtypes = [vp, c_int, c_int, c_int, c_int, vp, vp, c_int, c_int, vp, vp, vp, vp,
                                       c_size_t, vp]
    L.fq_flatten_quant_act_noalloc.argtypes = [vp, c_int, c_int, c_int, c_int, vp, vp, c_int, c_int, vp, vp, vp, vp]
    L.fq_noalloc_scratch_bytes.restype = c_size_t
    L.fq_noalloc_scratch_bytes.argtypes = []
    L.fq_peak_mfma.argtypes = [c_int, vp, c_size_t, c_int, ctypes.c_longlong, vp, vp, vp]
    L.fq_peak_copy.argtypes = [vp, vp, c_size_t, vp]
    L.fq_peak_gemm_ticks.argtypes = [vp]
    L.fq_peak_wall_clock_khz.argtypes = []
    L.fq_act_workspace_bytes.restype = c_size_t
    L.fq_act_workspace_bytes.argtypes = [c_int, c_int]
    for f in (L.fq_gemm_i8, L.fq_gemm_i4):
        f.argtypes = [vp, vp, c_int, c_int, c_int, vp, vp, vp, c_int, c_int, vp]
    for f in (L.fq_bmm_i8, L.fq_bmm_i4):
        f.argtypes = [vp, vp, c_int, c_int, c_int, c_int, ctypes.c_longlong, ctypes.c_longlong, vp, vp, vp, c_int,
                      c_int, ctypes.c_longlong, vp]
    for f in (L.fq_gemm_i8_bias, L.fq_gemm_i4_bias, L.fq_gemm_i4_e3m2):
        f.argtypes = [vp, vp, c_int, c_int, c_int, vp, vp, vp, vp, c_int, c_int, vp]
    L.fq_linear_fused_a_i8.argtypes = [vp, c_int, c_int, c_int, c_int, vp, vp, c_int, vp, vp, vp, c_int, vp, vp, c_int, c_int,
                                       vp, c_size_t, vp]
    L.fq_linear_bias.argtypes = [vp, c_int, c_int, c_int, c_int, vp, vp, c_int, vp, vp, vp, c_int, c_int, vp, vp,
                                 c_int, c_int, vp, c_size_t, vp]
    L.fq_linear.argtypes = [vp, c_int, c_int, c_int, c_int, vp, vp, c_int, vp, vp, c_int, c_int, vp, vp, c_int,
                            c_int, vp, c_size_t, vp]
    L.fq_linear_workspace_bytes.restype = c_size_t
    L.fq_linear_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int]
    L.fq_gemm_bf16.argtypes = [vp, vp, c_int, c_int, c_int, vp, c_int, vp]
    c_ll = ctypes.c_longlong
    L.fq_kv_append.argtypes = [vp, vp, vp, c_int, c_int, c_int, c_int, c_int, c_ll, c_ll, c_ll, vp, vp, c_int, c_int, vp, vp, c_int,
                               c_int, c_int, vp, c_ll, vp, c_ll, vp, vp, vp, vp, c_int, c_int, vp, c_int, vp]
    L.fq_attn_cache_workspace_bytes.restype = c_size_t
    L.fq_attn_cache_workspace_bytes.argtypes = [c_int] * 7
    L.fq_attn_cache.argtypes = [vp, c_int, c_int, c_int, c_int, c_int, c_ll, vp, vp, c_int, c_int, c_int, vp, vp, vp, vp, c_int, c_int, vp,
                                c_int, c_float, vp, c_ll, vp, c_size_t, vp]
    L.fq_attn_prompt.argtypes = [vp, vp, vp, c_int, c_int, c_int, c_int, c_int, c_int, c_ll, c_ll, c_ll, vp, vp, c_int, c_int, c_int, c_float, vp,
                                 c_ll, vp]
    for name in SYMBOLS:
        getattr(L, name)
    _lib = L
    return L


def _check(rc: int):
    if rc != FQ_OK:
        raise FqError(rc, lib().fq_last_error_string().decode())


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_codes = None


def _dtype_code(t) -> int:
    global _codes
    if _codes is None:
        torch = _torch()
        _codes = {torch.float32: FQ_F32, torch.float16: FQ_F16, torch.bfloat16: FQ_BF16, torch.int32: FQ_I32}
    return _codes[t.dtype]


_raw_stream = None


def _stream_on(stream, device) -> int:
    """_stream for callers that have the current device in hand."""
    if stream is not None:
        return getattr(stream, "cuda_stream", stream)
    global _raw_stream_of
    if _raw_stream_of is None:
        torch = _torch()
        _raw_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw_stream_of(device)


_raw_stream_of = None


def _stream(stream) -> int:
    """Raw handle of a stream, or of the current device's current stream.  The latter is read without building a
    torch.cuda.Stream object where torch offers that: about 2 us of a small call's 13."""
    global _raw_stream
    if stream is not None:
        return getattr(stream, "cuda_stream", stream)
    if _raw_stream is None:
        torch = _torch()
        get, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device
        _raw_stream = (lambda: get(device())) if get else (lambda: torch.cuda.current_stream().cuda_stream)
    return _raw_stream()


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev2d(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be 2-D with a contiguous last dimension")
    return t


# ------------------------------------------------------------------------------------------
# entry points (same names as the C ABI)
# ------------------------------------------------------------------------------------------
def fq_version() -> int:
    return lib().fq_version()


def fq_gemm_select(variant: int) -> None:
    _check(lib().fq_gemm_select(variant))


def fq_flatten_plan(chmax: np.ndarray, T: float, align: int = 32) -> Tuple[np.ndarray, np.ndarray, int, int]:
    """Host call.  Returns (src_idx int32 [Kpad], rep int32 [Kpad], Kprime, Kpad)."""
    chmax = np.ascontiguousarray(chmax, dtype=np.float32)
    K = chmax.shape[0]
    kp, kpad = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().fq_flatten_plan(chmax.ctypes.data, K, T, align, None, None, 0, ctypes.byref(kp), ctypes.byref(kpad)))
    src = np.empty(kpad.value, dtype=np.int32)
    rep = np.empty(kpad.value, dtype=np.int32)
    _check(lib().fq_flatten_plan(chmax.ctypes.data, K, T, align, src.ctypes.data, rep.ctypes.data, kpad.value,
                                 ctypes.byref(kp), ctypes.byref(kpad)))
    return src, rep, kp.value, kpad.value


def fq_flatten_plan_xw(chmax_x: np.ndarray, T_x: float, chmax_w: Optional[np.ndarray] = None, T_w: float = 1.0,
                       align: int = 32):
    """Host call.  Returns (src_idx, rep_x, rep_w, ord, Kprime, Kpad), int32 arrays of Kpad entries."""
    chmax_x = np.ascontiguousarray(chmax_x, dtype=np.float32)
    K = chmax_x.shape[0]
    cw = None if chmax_w is None else np.ascontiguousarray(chmax_w, dtype=np.float32)
    if cw is not None and cw.shape != chmax_x.shape:
        raise ValueError("chmax_x and chmax_w must have the same length")
    pw = None if cw is None else cw.ctypes.data
    kp, kpad = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().fq_flatten_plan_xw(chmax_x.ctypes.data, T_x, pw, T_w, K, align, None, None, None, None, 0,
                                    ctypes.byref(kp), ctypes.byref(kpad)))
    arrs = [np.empty(kpad.value, dtype=np.int32) for _ in range(4)]
    _check(lib().fq_flatten_plan_xw(chmax_x.ctypes.data, T_x, pw, T_w, K, align, *[a.ctypes.data for a in arrs],
                                    kpad.value, ctypes.byref(kp), ctypes.byref(kpad)))
    return arrs[0], arrs[1], arrs[2], arrs[3], kp.value, kpad.value


def fq_threshold_boxplot(chmax: np.ndarray, beta: float = 1.3) -> float:
    """Host call (Eq. 6-7).  Returns T as a Python float holding an fp32 value."""
    chmax = np.ascontiguousarray(chmax, dtype=np.float32)
    T = ctypes.c_float(0)
    _check(lib().fq_threshold_boxplot(chmax.ctypes.data, chmax.shape[0], beta, ctypes.byref(T)))
    return float(T.value)


def fq_smooth_scales(chmax_x: np.ndarray, chmax_w: np.ndarray, alpha: float = 0.5) -> np.ndarray:
    """Host call (Eq. 5).  Returns the fp32 smoothing factors s [K]."""
    chmax_x = np.ascontiguousarray(chmax_x, dtype=np.float32)
    chmax_w = np.ascontiguousarray(chmax_w, dtype=np.float32)
    if chmax_x.shape != chmax_w.shape:
        raise ValueError("chmax_x and chmax_w must have the same length")
    out = np.empty(chmax_x.shape[0], dtype=np.float32)
    _check(lib().fq_smooth_scales(chmax_x.ctypes.data, chmax_w.ctypes.data, chmax_x.shape[0], alpha, out.ctypes.data))
    return out


def fq_channel_absmax(X, chmax, accumulate: bool = False, stream=None) -> None:
    """chmax (fp32 [K], device) = per-channel max |X|, or the running maximum when accumulate is set."""
    _dev2d(X, "X")
    M, K = X.shape
    if chmax.numel() != K or _dtype_code(chmax) != FQ_F32 or not chmax.is_contiguous():
        raise ValueError("chmax must be a contiguous fp32 tensor of K elements")
    _check(lib().fq_channel_absmax(X.data_ptr(), _dtype_code(X), M, K, X.stride(0), int(bool(accumulate)),
                                   chmax.data_ptr(), _stream(stream)))


def fq_weights_workspace_bytes(K: int, Kpad: int) -> int:
    return lib().fq_weights_workspace_bytes(K, Kpad)


def fq_act_workspace_bytes(K: int, Kpad: int) -> int:
    return lib().fq_act_workspace_bytes(K, Kpad)


def fq_linear_workspace_bytes(M: int, K: int, Kpad: int, bits: int) -> int:
    return lib().fq_linear_workspace_bytes(M, K, Kpad, bits)


def fq_flatten_weights(W, src_idx, bits: int, Wq_out, s_w_out, workspace, stream=None) -> None:
    _dev2d(W, "W")
    N, K = W.shape
    Kpad = src_idx.numel()
    _check(lib().fq_flatten_weights(W.data_ptr(), _dtype_code(W), N, K, W.stride(0), src_idx.data_ptr(), Kpad, bits,
                                    Wq_out.data_ptr(), s_w_out.data_ptr(), workspace.data_ptr(),
                                    workspace.numel() * workspace.element_size(), _stream(stream)))


def fq_flatten_weights_split(W, src_idx, rep_w, bits: int, Wq_out, s_w_out, workspace, stream=None) -> None:
    _dev2d(W, "W")
    N, K = W.shape
    Kpad = src_idx.numel()
    _check(lib().fq_flatten_weights_split(W.data_ptr(), _dtype_code(W), N, K, W.stride(0), src_idx.data_ptr(),
                                          rep_w.data_ptr(), Kpad, bits, Wq_out.data_ptr(), s_w_out.data_ptr(),
                                          workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                          _stream(stream)))


def fq_flatten_quant_act_peel(X, src_idx, ord, bits: int, T: float, Xq_out, s_x_out, workspace, absmax_in=None,
                              stream=None) -> None:
    _dev2d(X, "X")
    M, K = X.shape
    Kpad = src_idx.numel()
    _check(lib().fq_flatten_quant_act_peel(X.data_ptr(), _dtype_code(X), M, K, X.stride(0), src_idx.data_ptr(),
                                           ord.data_ptr(), Kpad, bits, T, _ptr(absmax_in), Xq_out.data_ptr(),
                                           s_x_out.data_ptr(), workspace.data_ptr(),
                                           workspace.numel() * workspace.element_size(), _stream(stream)))


def fq_flatten_quant_act(X, src_idx, rep, bits: int, Xq_out, s_x_out, workspace, absmax_in=None, stream=None) -> None:
    _dev2d(X, "X")
    M, K = X.shape
    Kpad = src_idx.numel()
    _check(lib().fq_flatten_quant_act(X.data_ptr(), _dtype_code(X), M, K, X.stride(0), src_idx.data_ptr(),
                                      rep.data_ptr(), Kpad, bits, _ptr(absmax_in), Xq_out.data_ptr(),
                                      s_x_out.data_ptr(), workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), _stream(stream)))


def fq_noalloc_scratch_bytes() -> int:
    return int(lib().fq_noalloc_scratch_bytes())


def fq_flatten_quant_act_noalloc(X, src_idx, rep, bits: int, Xq_out, s_x_out, absmax_in=None, stream=None) -> None:
    """fq_flatten_quant_act with the workspace inside the library's device image (nothing is allocated)."""
    _dev2d(X, "X")
    M, K = X.shape
    Kpad = src_idx.numel()
    _check(lib().fq_flatten_quant_act_noalloc(X.data_ptr(), _dtype_code(X), M, K, X.stride(0), src_idx.data_ptr(),
                                              rep.data_ptr(), Kpad, bits, _ptr(absmax_in), Xq_out.data_ptr(),
                                              s_x_out.data_ptr(), _stream(stream)))


def fq_peak_mfma(kind: int, operands, blocks: int, iters: int, ticks_out, sink, stream=None) -> None:
    """MFMA-only issue loop (include/fq_peak.h).  operands: a device tensor of >= 64 KiB, or None for zeros."""
    nbytes = 0 if operands is None else operands.numel() * operands.element_size()
    _check(lib().fq_peak_mfma(kind, _ptr(operands), nbytes, blocks, iters, _ptr(ticks_out), sink.data_ptr(),
                              _stream(stream)))


def fq_peak_gemm_ticks(ticks) -> None:
    """ticks: int64 device tensor [2] the GEMM kernels launched from this thread add their clock ticks to, or None."""
    _check(lib().fq_peak_gemm_ticks(_ptr(ticks)))


def fq_peak_wall_clock_khz() -> int:
    return int(lib().fq_peak_wall_clock_khz())


def fq_peak_copy(src, dst, stream=None) -> None:
    """Plain device copy of src into dst (same byte size, a multiple of 16)."""
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    _check(lib().fq_peak_copy(src.data_ptr(), dst.data_ptr(), nbytes, _stream(stream)))


def _gemm(fn, Xq, Wq, M, N, Kpad, s_x, s_w, Y, stream):
    _dev2d(Y, "Y")
    _check(fn(Xq.data_ptr(), Wq.data_ptr(), M, N, Kpad, _ptr(s_x), _ptr(s_w), Y.data_ptr(), _dtype_code(Y),
              Y.stride(0), _stream(stream)))


def fq_gemm_i8(Xq, Wq, s_x, s_w, Y, stream=None) -> None:
    """Xq int8 [M, Kpad], Wq int8 [N, Kpad] -> Y [M, N] (f32/f16/bf16, or int32 raw accumulators)."""
    M, Kpad = Xq.shape
    N = Wq.shape[0]
    _gemm(lib().fq_gemm_i8, Xq, Wq, M, N, Kpad, s_x, s_w, Y, stream)


def _gemm_bias(fn, Xq, Wq, M, N, Kpad, s_x, s_w, bias, Y, stream):
    _dev2d(Y, "Y")
    if bias is not None and (bias.numel() != N or _dtype_code(bias) != FQ_F32 or not bias.is_contiguous()):
        raise ValueError("bias must be a contiguous fp32 tensor of N elements")
    _check(fn(Xq.data_ptr(), Wq.data_ptr(), M, N, Kpad, _ptr(s_x), _ptr(s_w), _ptr(bias), Y.data_ptr(), _dtype_code(Y),
              Y.stride(0), _stream(stream)))


def fq_gemm_i8_bias(Xq, Wq, s_x, s_w, bias, Y, stream=None) -> None:
    M, Kpad = Xq.shape
    _gemm_bias(lib().fq_gemm_i8_bias, Xq, Wq, M, Wq.shape[0], Kpad, s_x, s_w, bias, Y, stream)


def fq_gemm_i4_bias(Xq, Wq, s_x, s_w, bias, Y, stream=None) -> None:
    M, half = Xq.shape
    _gemm_bias(lib().fq_gemm_i4_bias, Xq, Wq, M, Wq.shape[0], 2 * half, s_x, s_w, bias, Y, stream)


def fq_gemm_i4_e3m2(Xq, Wq, s_x, s_w, bias, Y, stream=None) -> None:
    """Xq uint8 [Kpad / 128, M, 96], Wq uint8 [Kpad / 128, N, 96] (k-blocked 6-bit E3M2 codes of 4-bit values)
    -> Y [M, N]."""
    if Xq.dim() != 3 or Wq.dim() != 3 or Xq.shape[2] != 96 or Wq.shape[2] != 96 or Xq.shape[0] != Wq.shape[0]:
        raise ValueError("E3M2 operands are [Kpad / 128, rows, 96] byte arrays")
    if not (Xq.is_contiguous() and Wq.is_contiguous()):
        raise ValueError("E3M2 operands must be contiguous")
    _gemm_bias(lib().fq_gemm_i4_e3m2, Xq, Wq, Xq.shape[1], Wq.shape[1], 128 * Xq.shape[0], s_x, s_w, bias, Y, stream)


def fq_linear_bias(X, src_idx, rep, Wq, s_w, bias, bits: int, Y, workspace, absmax_in=None, stream=None) -> None:
    _dev2d(X, "X")
    _dev2d(Y, "Y")
    M, K = X.shape
    Kpad = src_idx.numel()
    N = Wq.shape[1] if Wq.dim() == 3 else Wq.shape[0]      # E3M2 weights are [Kpad / 128, N, 96]
    if bias is not None and (bias.numel() != N or _dtype_code(bias) != FQ_F32 or not bias.is_contiguous()):
        raise ValueError("bias must be a contiguous fp32 tensor of N elements")
    _check(lib().fq_linear_bias(X.data_ptr(), _dtype_code(X), M, K, X.stride(0), src_idx.data_ptr(), rep.data_ptr(),
                                Kpad, Wq.data_ptr(), s_w.data_ptr(), _ptr(bias), N, bits, _ptr(absmax_in), Y.data_ptr(),
                                _dtype_code(Y), Y.stride(0), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), _stream(stream)))


def fq_linear_fused_a_i8(X, src_idx, rep, Wq, s_w, Y, workspace, bias=None, absmax_in=None, stream=None) -> None:
    """The INT8 layer with flatten + quantize fused into the GEMM's A-operand load: X bf16 [M, K], Wq int8 [N, Kpad]
    -> Y [M, N]; workspace of fq_act_workspace_bytes(K, Kpad) bytes."""
    _dev2d(X, "X")
    _dev2d(Y, "Y")
    M, K = X.shape
    Kpad = src_idx.numel()
    N = Wq.shape[0]
    if bias is not None and (bias.numel() != N or _dtype_code(bias) != FQ_F32 or not bias.is_contiguous()):
        raise ValueError("bias must be a contiguous fp32 tensor of N elements")
    _check(lib().fq_linear_fused_a_i8(X.data_ptr(), _dtype_code(X), M, K, X.stride(0), src_idx.data_ptr(), rep.data_ptr(),
                                      Kpad, Wq.data_ptr(), _ptr(s_w), _ptr(bias), N, _ptr(absmax_in), Y.data_ptr(),
                                      _dtype_code(Y), Y.stride(0), workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), _stream(stream)))


def fq_gemm_i4(Xq, Wq, s_x, s_w, Y, stream=None) -> None:
    """Xq uint8 [M, Kpad/2], Wq uint8 [N, Kpad/2] (packed nibbles) -> Y [M, N]."""
    M, half = Xq.shape
    N = Wq.shape[0]
    _gemm(lib().fq_gemm_i4, Xq, Wq, M, N, 2 * half, s_x, s_w, Y, stream)


def _bmm(fn, Aq, Bq, Kpad, s_a, s_b, Y, stream):
    for t, name in ((Aq, "Aq"), (Bq, "Bq"), (Y, "Y")):
        if not t.is_cuda or t.dim() != 3 or t.stride(2) != 1:
            raise ValueError(f"{name} must be a 3-D device tensor with a contiguous last dimension")
    batch, M, rowbytes = Aq.shape
    N = Bq.shape[1]
    if Bq.shape[0] != batch or Bq.shape[2] != rowbytes or Y.shape != (batch, M, N):
        raise ValueError("shape mismatch between Aq, Bq and Y")
    if Aq.stride(1) != rowbytes or Bq.stride(1) != rowbytes:
        raise ValueError("operand rows must be dense")
    _check(fn(Aq.data_ptr(), Bq.data_ptr(), batch, M, N, Kpad, Aq.stride(0), Bq.stride(0), _ptr(s_a), _ptr(s_b),
              Y.data_ptr(), _dtype_code(Y), Y.stride(1), Y.stride(0), _stream(stream)))


def fq_bmm_i8(Aq, Bq, s_a, s_b, Y, stream=None) -> None:
    """Aq int8 [batch, M, Kpad], Bq int8 [batch, N, Kpad] -> Y [batch, M, N]."""
    _bmm(lib().fq_bmm_i8, Aq, Bq, Aq.shape[2], s_a, s_b, Y, stream)


def fq_bmm_i4(Aq, Bq, s_a, s_b, Y, stream=None) -> None:
    """Aq uint8 [batch, M, Kpad/2], Bq uint8 [batch, N, Kpad/2] (packed nibbles) -> Y [batch, M, N]."""
    _bmm(lib().fq_bmm_i4, Aq, Bq, 2 * Aq.shape[2], s_a, s_b, Y, stream)


def fq_linear(X, src_idx, rep, Wq, s_w, bits: int, Y, workspace, absmax_in=None, stream=None) -> None:
    _dev2d(X, "X")
    _dev2d(Y, "Y")
    M, K = X.shape
    Kpad = src_idx.numel()
    N = Wq.shape[1] if Wq.dim() == 3 else Wq.shape[0]      # E3M2 weights are [Kpad / 128, N, 96]
    _check(lib().fq_linear(X.data_ptr(), _dtype_code(X), M, K, X.stride(0), src_idx.data_ptr(), rep.data_ptr(), Kpad,
                           Wq.data_ptr(), s_w.data_ptr(), N, bits, _ptr(absmax_in), Y.data_ptr(), _dtype_code(Y),
                           Y.stride(0), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                           _stream(stream)))


def fq_gemm_bf16(X, W, Y, stream=None) -> None:
    _dev2d(X, "X")
    _dev2d(W, "W")
    _dev2d(Y, "Y")
    M, K = X.shape
    N = W.shape[0]
    if X.stride(0) != K or W.stride(0) != K:
        raise ValueError("fq_gemm_bf16 needs densely packed rows")
    _check(lib().fq_gemm_bf16(X.data_ptr(), W.data_ptr(), M, N, K, Y.data_ptr(), Y.stride(0), _stream(stream)))


# ------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------
# The checks of these calls read each tensor's shape, strides and type once: of a small call's 14 us they were 8.
def _here() -> int:
    """The current device, whose stream the kernels go to."""
    global _get_device
    if _get_device is None:
        torch = _torch()
        _get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _get_device()


_get_device = None


def _packed(t, name, here, shape=None, dtype=None):
    """(shape, token stride) of a packed [tokens, heads, head_dim] tensor with dense heads on device `here`."""
    if t.get_device() != here:
        raise ValueError(f"{name} is on {t.device}: it must be on the current device, cuda:{here}")
    got, strides = t.shape, t.stride()
    if len(got) != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    tokens, heads, dim = got
    if shape is not None and (got != shape or t.dtype != dtype):
        raise ValueError(f"{name} must have the shape and type {tuple(shape)}, {dtype}")
    if tokens and ((dim > 1 and strides[2] != 1) or (heads > 1 and strides[1] != dim)):
        raise ValueError(f"{name} must have dense heads: only its token stride is free")
    return got, strides[0] if tokens > 1 else heads * dim


def _array(t, name, here, dtype, shape):
    """Address of a contiguous tensor of that type and shape on device `here`."""
    if t.dtype is not dtype or t.get_device() != here or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the current device, cuda:{here}; it is {t.dtype}, "
                         f"{tuple(t.shape)}, on {t.device}")
    return t.data_ptr()


def _cache(k_cache, v_cache, k_scale, v_scale, page_table, batch, dim, here):
    """(heads_kv, addresses, pages, page size, address of the table, its columns) of a paged cache whose tensors fit together."""
    torch = _torch()
    if k_cache.dim() != 4:
        raise ValueError("k_cache is [pages, heads_kv, page_size, head_dim]")
    pages, heads, size, _ = k_cache.shape
    width = page_table.shape[-1]
    return (heads, (_array(k_cache, "k_cache", here, torch.int8, (pages, heads, size, dim)), _array(v_cache, "v_cache", here, torch.int8, (pages, heads, dim, size)),
                    _array(k_scale, "k_scale", here, torch.float32, (pages, heads)), _array(v_scale, "v_scale", here, torch.float32, (pages, heads)), pages, size,
                    _array(page_table, "page_table", here, torch.int32, (batch, width)), width))


def fq_kv_append(Q, K, V, cu_new, past, max_new: int, k_cache, v_cache, k_scale, v_scale, page_table, rope_cos=None, rope_sin=None,
                 interleaved: bool = False, Q_out=None, K_out=None, stream=None) -> None:
    """Rotate Q [tokens, heads_q, head_dim] into Q_out and K [tokens, heads_kv, head_dim] into K_out (either None: not wanted), and
    store K and V at positions past[b] .. of each sequence in the paged 8-bit cache, whose codes and scales are updated in place.
    rope_cos, rope_sin fp32 [positions, rope_dim / 2], or None: no rotation."""
    torch, here = _torch(), _here()
    shape, ldk = _packed(K, "K", here)
    dtype = K.dtype
    ldv = _packed(V, "V", here, shape, dtype)[1]
    tokens, heads_kv, dim = shape
    q = q_out = k_out = cos = sin = None
    heads_q, ldq, ldqo, ldko, rows, half = heads_kv, heads_kv * dim, heads_kv * dim, heads_kv * dim, 0, 0
    if Q_out is not None:
        if Q is None:
            raise ValueError("Q_out without Q")
        q_shape, ldq = _packed(Q, "Q", here)
        heads_q = q_shape[1]
        if q_shape[0] != tokens or q_shape[2] != dim or Q.dtype != dtype:
            raise ValueError("Q must have K's tokens, head_dim and type")
        ldqo = _packed(Q_out, "Q_out", here, q_shape, dtype)[1]
        q, q_out = Q.data_ptr(), Q_out.data_ptr()
    if K_out is not None:
        ldko, k_out = _packed(K_out, "K_out", here, shape, dtype)[1], K_out.data_ptr()
    batch = past.numel()
    heads, cache = _cache(k_cache, v_cache, k_scale, v_scale, page_table, batch, dim, here)
    if heads != heads_kv:
        raise ValueError(f"K has {heads_kv} heads, the cache {heads}")
    if (rope_cos is None) != (rope_sin is None):
        raise ValueError("rope_cos and rope_sin go together")
    if rope_cos is not None:
        if rope_cos.dim() != 2:
            raise ValueError("rope_cos is [positions, rope_dim / 2]")
        rows, half = rope_cos.shape
        cos, sin = _array(rope_cos, "rope_cos", here, torch.float32, (rows, half)), _array(rope_sin, "rope_sin", here, torch.float32, (rows, half))
    rc = (_lib or lib()).fq_kv_append(q, K.data_ptr(), V.data_ptr(), _dtype_code(K), tokens, heads_q, heads_kv, dim, ldq, ldk, ldv,
                                      _array(cu_new, "cu_new", here, torch.int32, (batch + 1,)), _array(past, "past", here, torch.int32, (batch,)), batch, max_new,
                                      cos, sin, rows, 2 * half, 1 if interleaved else 0, q_out, ldqo, k_out, ldko, *cache, _stream_on(stream, here))
    if rc:
        _check(rc)


def fq_attn_cache_workspace_bytes(batch: int, tokens: int, max_q: int, max_len: int, heads_q: int, heads_kv: int, head_dim: int) -> int:
    return lib().fq_attn_cache_workspace_bytes(batch, tokens, max_q, max_len, heads_q, heads_kv, head_dim)


def fq_attn_cache(Q, cu_q, lens, max_q: int, max_len: int, k_cache, v_cache, k_scale, v_scale, page_table, scale: float, Y, workspace,
                  stream=None) -> None:
    """Y = causal attention of Q [tokens, heads_q, head_dim], the last tokens of each sequence (rows cu_q[b] .. cu_q[b + 1] - 1), over the
    lens[b] tokens that the paged 8-bit cache holds of it."""
    torch, here = _torch(), _here()
    shape, ldq = _packed(Q, "Q", here)
    ldy = _packed(Y, "Y", here, shape, Q.dtype)[1]
    tokens, heads_q, dim = shape
    batch = lens.numel()
    heads_kv, cache = _cache(k_cache, v_cache, k_scale, v_scale, page_table, batch, dim, here)
    if workspace.get_device() != here or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on the current device, cuda:{here}")
    rc = (_lib or lib()).fq_attn_cache(Q.data_ptr(), _dtype_code(Q), tokens, heads_q, heads_kv, dim, ldq, _array(cu_q, "cu_q", here, torch.int32, (batch + 1,)),
                                       _array(lens, "lens", here, torch.int32, (batch,)), batch, max_q, max_len, *cache, scale, Y.data_ptr(), ldy,
                                       workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_on(stream, here))
    if rc:
        _check(rc)


def fq_attn_prompt(Q, K, V, cu_q, cu_k, max_q: int, scale: float, Y, causal: bool = True, stream=None) -> None:
    """Y = attention of packed queries Q [tokens_q, heads_q, head_dim] over packed K, V [tokens_k, heads_kv, head_dim], sequence by
    sequence (rows cu_q[b] .. and cu_k[b] .. belong together); causal: the last query of a sequence sees its last key."""
    torch, here = _torch(), _here()
    shape, ldq = _packed(Q, "Q", here)
    ldy = _packed(Y, "Y", here, shape, Q.dtype)[1]
    k_shape, ldk = _packed(K, "K", here)
    ldv = _packed(V, "V", here, k_shape, K.dtype)[1]
    tokens_q, heads_q, dim = shape
    tokens_k, heads_kv, dim_k = k_shape
    if dim_k != dim or K.dtype != Q.dtype:
        raise ValueError("Q, K and V must have the same head_dim and type")
    batch = cu_q.numel() - 1
    rc = (_lib or lib()).fq_attn_prompt(Q.data_ptr(), K.data_ptr(), V.data_ptr(), _dtype_code(Q), tokens_q, tokens_k, heads_q, heads_kv, dim, ldq, ldk, ldv,
                                        _array(cu_q, "cu_q", here, torch.int32, (batch + 1,)), _array(cu_k, "cu_k", here, torch.int32, (batch + 1,)), batch, max_q,
                                        1 if causal else 0, scale, Y.data_ptr(), ldy, _stream_on(stream, here))
    if rc:
        _check(rc)
