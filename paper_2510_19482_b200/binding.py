"""ctypes binding: one Python function per C entry point, same names, argument marshalling only."""

from __future__ import annotations

import ctypes
import os
from ctypes import c_char_p, c_int, c_longlong, c_size_t, c_uint, c_ulonglong, c_void_p

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

FLAG_SKIP_OFFSET = 0x1
FLAG_OFFSET_ONLY = 0x2
FLAG_OUT_F32 = 0x4
FLAG_ACCUMULATE = 0x8
FLAG_PLAIN_G4 = 0x10
FLAG_CLUSTER_REDUCE = 0x20
FLAG_MIRROR = 0x40
FLAG_LUT_ONLY = 0x80
FLAG_TABLE_F16 = 0x100
FLAG_TABLE_I8 = 0x200

# elutq_gemm_kernel
KERNEL_DECODE, KERNEL_LOOK_UP, KERNEL_FRAGMENT, KERNEL_TENSOR_MEMORY, KERNEL_SHARED_MEMORY = range(5)

MX4_MXFP4, MX4_NVFP4 = 0, 1
MX4_FLAG_SWIGLU = 0x1
TYPE_F16, TYPE_BF16, TYPE_F32 = 0, 1, 2


class GemvCall(ctypes.Structure):
    """elutq_gemv_call: one M = 1 call of a chain."""
    _fields_ = [("X", c_void_p), ("packed", c_void_p), ("Y", c_void_p), ("N", c_int), ("K", c_int), ("flags", c_uint)]


class ElutqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().elutq_status_string(status).decode()
        extra = f" (cudaError {lib().elutq_last_cuda_error()})" if status == -6 else ""
        super().__init__(f"{where}: {msg}{extra} [{status}]")


def library_path() -> str:
    return os.path.join(_HERE, "libelutq.so")


_SIGNATURES = {
    "elutq_status_string": (c_char_p, [c_int]),
    "elutq_last_cuda_error": (c_int, []),
    "elutq_packed_bytes": (c_int, [c_int, c_int, c_int, c_int, ctypes.POINTER(c_size_t)]),
    "elutq_pack": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_size_t, c_void_p]),
    "elutq_unpack": (c_int, [c_void_p, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p]),
    "elutq_describe": (c_int, [c_void_p, c_int, c_int, ctypes.POINTER(c_int), ctypes.POINTER(c_int)]),
    "elutq_forget": (c_int, [c_void_p]),
    "elutq_workspace_bytes": (c_int, [c_int, c_int, c_int, ctypes.POINTER(c_size_t)]),
    "elutq_workspace_init": (c_int, [c_void_p, c_size_t, c_void_p]),
    "elutq_lut_gemm": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]),
    "elutq_lut_gemm_bias": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p]),
    "elutq_lut_gemm_f32": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_uint, c_void_p]),
    "elutq_lut_gemm_ws": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_uint, c_void_p, c_size_t, c_void_p]),
    "elutq_lut_gemm_host": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]),
    "elutq_lut_gemm_static": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]),
    "elutq_takes_tensor_path": (c_int, [c_int, c_int, c_int, c_int, c_uint]),
    "elutq_gemm_kernel": (c_int, [c_int, c_int, c_int, c_int, c_int, c_uint]),
    "elutq_hlq_fit": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "elutq_mx4_bytes": (c_int, [c_int, c_int, c_int, ctypes.POINTER(c_size_t), ctypes.POINTER(c_size_t)]),
    "elutq_mx4_quantize": (c_int, [c_void_p, c_int, c_int, c_longlong, c_int, c_int, c_int, c_uint, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_void_p]),
    "elutq_mx4_dequantize": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p, c_int, c_void_p]),
    "elutq_mx4_gemm": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p]),
    "elutq_mx4_gemm_grouped": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p]),
    "elutq_mx4_test_wait_expiry": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_uint, c_void_p]),
    "elutq_chain_plan_bytes": (c_int, [ctypes.POINTER(GemvCall), c_int, ctypes.POINTER(c_size_t)]),
    "elutq_chain_plan": (c_int, [ctypes.POINTER(GemvCall), c_int, c_void_p, c_size_t, c_void_p]),
    "elutq_chain_run": (c_int, [c_void_p, c_int, c_void_p]),
    "elutq_chain_run_opts": (c_int, [c_void_p, c_int, c_uint, c_void_p]),
    "elutq_chain_run_host": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_size_t, c_void_p, c_void_p, c_size_t, c_void_p]),
    "elutq_chain_status": (c_int, [c_void_p, c_void_p, ctypes.POINTER(c_int)]),
    "elutq_chain_forget": (c_int, [c_void_p]),
    "elutq_chain_shares": (c_int, [c_int, c_int, c_int, c_int, c_int, ctypes.POINTER(c_int), ctypes.POINTER(c_int)]),
    "elutq_device_status": (c_int, [c_void_p, ctypes.POINTER(c_int)]),
    "elutq_launch_count": (c_ulonglong, []),
    "elutq_release_scratch": (c_int, []),
    "elutq_test_wait_expiry": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_uint, c_void_p]),
    "elutq_reserve": (c_int, [c_int, c_int, c_int, c_void_p]),
    "elutq_scratch_address": (c_int, [c_void_p, c_int, ctypes.POINTER(c_void_p), ctypes.POINTER(c_size_t)]),
}


def lib() -> ctypes.CDLL:
    """Load libelutq.so (built in-tree by `paper_2510_19482_b200.build`); raises if it is missing."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} not found: build it with `python -m paper_2510_19482_b200.build` "
                              "(there is no CPU fallback)")
        handle = ctypes.CDLL(path)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = handle
    return _LIB


def _check(status: int, where: str) -> None:
    if status != 0:
        raise ElutqError(status, where)


def _ptr(t) -> int:
    """Raw address of a torch tensor (device or host); None -> NULL."""
    return 0 if t is None else t.data_ptr()


_CURRENT = None      # torch's current device, and its current stream's address


def _stream(stream) -> int:
    """Address of a stream; None = torch's current one (its raw handle: building a torch.cuda.Stream takes 3 us a call)."""
    global _CURRENT
    if stream is None:
        if _CURRENT is None:
            import torch
            raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
            _CURRENT = (torch.cuda.current_device, raw or (lambda device: torch.cuda.current_stream(device).cuda_stream))
        device, raw = _CURRENT
        return raw(device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def elutq_status_string(status: int) -> str:
    return lib().elutq_status_string(status).decode()


def elutq_last_cuda_error() -> int:
    return lib().elutq_last_cuda_error()


def elutq_launch_count() -> int:
    return int(lib().elutq_launch_count())


def elutq_release_scratch() -> None:
    _check(lib().elutq_release_scratch(), "elutq_release_scratch")


def elutq_packed_bytes(q: int, G: int, N: int, K: int) -> int:
    out = c_size_t(0)
    _check(lib().elutq_packed_bytes(q, G, N, K, ctypes.byref(out)), "elutq_packed_bytes")
    return out.value


def elutq_pack(planes, scales, offsets, q: int, G: int, N: int, K: int, packed=None, stream=None):
    """planes uint8 [q,N,K], scales fp16 [N,K/G,q], offsets fp16 [N,K/G] (CUDA tensors) -> packed uint8 blob."""
    import torch
    if packed is None:
        packed = torch.empty(elutq_packed_bytes(q, G, N, K), dtype=torch.uint8, device=planes.device)
    _check(lib().elutq_pack(_ptr(planes), _ptr(scales), _ptr(offsets), q, G, N, K,
                            _ptr(packed), packed.numel() * packed.element_size(), _stream(stream)), "elutq_pack")
    return packed


def elutq_unpack(packed, N: int, K: int, planes, scales, offsets, stream=None) -> None:
    _check(lib().elutq_unpack(_ptr(packed), N, K, _ptr(planes), _ptr(scales), _ptr(offsets), _stream(stream)),
           "elutq_unpack")


def elutq_describe(packed, N: int, K: int):
    q, G = c_int(0), c_int(0)
    _check(lib().elutq_describe(_ptr(packed), N, K, ctypes.byref(q), ctypes.byref(G)), "elutq_describe")
    return q.value, G.value


def elutq_forget(packed) -> None:
    _check(lib().elutq_forget(_ptr(packed)), "elutq_forget")


def elutq_workspace_bytes(M: int, N: int, K: int) -> int:
    out = c_size_t(0)
    _check(lib().elutq_workspace_bytes(M, N, K, ctypes.byref(out)), "elutq_workspace_bytes")
    return out.value


def elutq_workspace_init(workspace, stream=None) -> None:
    _check(lib().elutq_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "elutq_workspace_init")


def elutq_lut_gemm(X, packed, Y, M: int, N: int, K: int, stream=None) -> None:
    _check(lib().elutq_lut_gemm(_ptr(X), _ptr(packed), _ptr(Y), M, N, K, _stream(stream)), "elutq_lut_gemm")


def elutq_lut_gemm_bias(X, packed, Y, M: int, N: int, K: int, accumulate: bool = False, stream=None) -> None:
    _check(lib().elutq_lut_gemm_bias(_ptr(X), _ptr(packed), _ptr(Y), M, N, K, int(bool(accumulate)), _stream(stream)),
           "elutq_lut_gemm_bias")


def elutq_lut_gemm_f32(X, packed, Y, M: int, N: int, K: int, flags: int = 0, stream=None) -> None:
    _check(lib().elutq_lut_gemm_f32(_ptr(X), _ptr(packed), _ptr(Y), M, N, K, flags, _stream(stream)),
           "elutq_lut_gemm_f32")


def elutq_lut_gemm_ws(X, packed, Y, M: int, N: int, K: int, flags: int, workspace, stream=None) -> None:
    _check(lib().elutq_lut_gemm_ws(_ptr(X), _ptr(packed), _ptr(Y), M, N, K, flags, _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)), "elutq_lut_gemm_ws")


def elutq_lut_gemm_host(X_host, packed, Y_host, M: int, N: int, K: int, stream=None) -> None:
    _check(lib().elutq_lut_gemm_host(_ptr(X_host), _ptr(packed), _ptr(Y_host), M, N, K, _stream(stream)),
           "elutq_lut_gemm_host")


def elutq_takes_tensor_path(M: int, N: int, K: int, G: int = 128, flags: int = 0) -> bool:
    """True when elutq_lut_gemm runs this shape on the tensor-core path whatever q is (host-only)."""
    return bool(lib().elutq_takes_tensor_path(M, N, K, G, flags))


def elutq_gemm_kernel(M: int, N: int, K: int, q: int, G: int = 128, flags: int = 0) -> int:
    """The kernel a call of this shape runs on (KERNEL_...); host-only."""
    kernel = lib().elutq_gemm_kernel(M, N, K, q, G, flags)
    if kernel < 0:
        _check(kernel, "elutq_gemm_kernel")
    return kernel


def elutq_lut_gemm_static(X, packed, Y, M: int, N: int, K: int, stream=None) -> None:
    """elutq_lut_gemm for callers that must not allocate: scratch is a fixed 4 MiB array inside the library."""
    _check(lib().elutq_lut_gemm_static(_ptr(X), _ptr(packed), _ptr(Y), M, N, K, _stream(stream)),
           "elutq_lut_gemm_static")


def elutq_hlq_fit(W, q: int, G: int, t_max: int = 10, trace: bool = False, stream=None):
    """Algorithm 1 on a CUDA fp16 matrix W [N, K] -> (planes uint8 [q,N,K], scales fp16 [N,K/G,q],
    offsets fp16 [N,K/G]) and, with trace=True, the per-group squared error [t_max+1, N*K/G] (fp64)."""
    import torch
    N, K = W.shape
    planes = torch.empty((q, N, K), dtype=torch.uint8, device=W.device)
    scales = torch.empty((N, K // G, q), dtype=torch.float16, device=W.device)
    offsets = torch.empty((N, K // G), dtype=torch.float16, device=W.device)
    tr = torch.empty((t_max + 1, N * (K // G)), dtype=torch.float64, device=W.device) if trace else None
    _check(lib().elutq_hlq_fit(_ptr(W), q, G, N, K, t_max, _ptr(planes), _ptr(scales), _ptr(offsets),
                               _ptr(tr) if trace else None, _stream(stream)), "elutq_hlq_fit")
    return (planes, scales, offsets, tr) if trace else (planes, scales, offsets)


_TORCH = None


def _torch():
    """(torch, {dtype: ELUTQ_TYPE_}, function: current device, function: a device's current stream)"""
    global _TORCH
    if _TORCH is None:
        import torch
        device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
        _TORCH = (torch, {torch.float16: TYPE_F16, torch.bfloat16: TYPE_BF16, torch.float32: TYPE_F32}, device, raw)
    return _TORCH


def _refuse(where: str, wanted: str, *tensors):
    got = ", ".join("nothing" if t is None else f"{t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ' with gaps'}" for t in tensors)
    raise ElutqError(-1, f"{where} ({wanted}, dense and on the current CUDA device; got {got})")


def _small(where: str, name: str, t, dtype, numel: int, device: int) -> int:
    """Address of a small operand; None -> NULL."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.numel() < numel or not t.is_contiguous() or t.get_device() != device:
        _refuse(where, f"{name}: {numel} values of {dtype} wanted", t)
    return t.data_ptr()


def elutq_mx4_bytes(fmt: int, rows: int, K: int):
    """(bytes of the codes, bytes of the scales) of a matrix."""
    codes, scales = c_size_t(0), c_size_t(0)
    _check(lib().elutq_mx4_bytes(fmt, rows, K, ctypes.byref(codes), ctypes.byref(scales)), "elutq_mx4_bytes")
    return codes.value, scales.value


def _mx4_block(fmt: int) -> int:
    return 32 if fmt == MX4_MXFP4 else 16


def elutq_mx4_quantize(X, rows: int, K: int, fmt: int, codes=None, scales=None, flags: int = 0, prescale=None, index=None, index_div: int = 1,
                       n_rows=None, stream=None):
    """X fp16, bf16 or fp32 [x_rows, K] (or [x_rows, 2 K], SwiGLU), unit stride along a row -> (codes uint8 [rows, K/2], scales uint8 [rows, K/B]).
    index int32 [rows], n_rows int32 [1], prescale fp32 [1]."""
    where = "elutq_mx4_quantize"
    torch, types, current, raw = _torch()
    d, shape, stride = X.get_device(), X.shape, X.stride()
    width = 2 * K if flags & MX4_FLAG_SWIGLU else K
    if len(stride) != 2 or stride[1] != 1 or shape[1] < width or d < 0 or d != current():
        _refuse(where, f"X: [x_rows, {width}] with unit stride along a row wanted", X)
    half, blocks = K // 2, K // _mx4_block(fmt)
    if codes is None:
        codes = X.new_empty((rows, half), dtype=torch.uint8)
    elif codes.nbytes != rows * half or not codes.is_contiguous() or codes.get_device() != d:
        _refuse(where, f"codes: {rows * half} bytes wanted", codes)
    if scales is None:
        scales = X.new_empty((rows, blocks), dtype=torch.uint8)
    elif scales.nbytes != rows * blocks or not scales.is_contiguous() or scales.get_device() != d:
        _refuse(where, f"scales: {rows * blocks} bytes wanted", scales)
    _check(lib().elutq_mx4_quantize(X.data_ptr(), types.get(X.dtype, -1), shape[0], stride[0] if shape[0] > 1 else width, rows, K, fmt, flags,
                                    _small(where, "prescale", prescale, torch.float32, 1, d), _small(where, "index", index, torch.int32, rows, d), index_div,
                                    _small(where, "n_rows", n_rows, torch.int32, 1, d), codes.data_ptr(), scales.data_ptr(),
                                    raw(d) if stream is None else _stream(stream)), where)
    return codes, scales


def elutq_mx4_dequantize(codes, scales, Y, rows: int, K: int, fmt: int, alpha=None, stream=None) -> None:
    """codes, scales -> Y fp16, bf16 or fp32 [rows, K]; alpha fp32 [1]."""
    where = "elutq_mx4_dequantize"
    torch, types, current, raw = _torch()
    d = Y.get_device()
    if (d < 0 or d != current() or codes.nbytes != rows * (K // 2) or not codes.is_contiguous() or codes.get_device() != d or
            scales.nbytes != rows * (K // _mx4_block(fmt)) or not scales.is_contiguous() or scales.get_device() != d or
            Y.numel() != rows * K or not Y.is_contiguous()):
        _refuse(where, f"codes, scales: {rows * (K // 2)} and {rows * (K // _mx4_block(fmt))} bytes, Y: {rows} x {K} values wanted", codes, scales, Y)
    _check(lib().elutq_mx4_dequantize(codes.data_ptr(), scales.data_ptr(), rows, K, fmt, _small(where, "alpha", alpha, torch.float32, 1, d),
                                      Y.data_ptr(), types.get(Y.dtype, -1), raw(d) if stream is None else _stream(stream)), where)


_PRODUCTS = None


def _products():
    """What a call of the products needs, looked up once: their C functions, ELUTQ_TYPE_ by dtype, the current device and a device's current stream."""
    global _PRODUCTS
    if _PRODUCTS is None:
        _, types, current, raw = _torch()
        _PRODUCTS = (lib().elutq_mx4_gemm, lib().elutq_mx4_gemm_grouped, types, current, raw)
    return _PRODUCTS


def _mx4_check(where, x_codes, x_scales, w_codes, w_scales, Y, M, N, K, rows, fmt):
    """The product's operands and result are dense, of the right size (codes and scales are bytes, whatever type they go by) and on the current device."""
    d, half, blocks = Y.get_device(), K // 2, K // 32 if fmt == MX4_MXFP4 else K // 16
    if (d < 0 or d != _PRODUCTS[3]() or Y.numel() != M * N or not Y.is_contiguous() or
            x_codes.nbytes != M * half or not x_codes.is_contiguous() or x_codes.get_device() != d or
            x_scales.nbytes != M * blocks or not x_scales.is_contiguous() or x_scales.get_device() != d or
            w_codes.nbytes != rows * half or not w_codes.is_contiguous() or w_codes.get_device() != d or
            w_scales.nbytes != rows * blocks or not w_scales.is_contiguous() or w_scales.get_device() != d):
        _refuse(where, f"X: {M * half} and {M * blocks} bytes, W: {rows * half} and {rows * blocks} bytes, Y: {M} x {N} values wanted",
                x_codes, x_scales, w_codes, w_scales, Y)
    return d


def elutq_mx4_gemm(x_codes, x_scales, w_codes, w_scales, Y, M: int, N: int, K: int, fmt: int, alpha=None, stream=None) -> None:
    """Y fp16, bf16 or fp32 [M, N] = alpha X W^T; codes and scales of X [M, K] and W [N, K]; alpha fp32 [1]."""
    gemm, _, types, _, raw = _PRODUCTS or _products()
    d = _mx4_check("elutq_mx4_gemm", x_codes, x_scales, w_codes, w_scales, Y, M, N, K, N, fmt)
    status = gemm(x_codes.data_ptr(), x_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), Y.data_ptr(), types.get(Y.dtype, -1), M, N, K, fmt,
                  0 if alpha is None else _small("elutq_mx4_gemm", "alpha", alpha, _TORCH[0].float32, 1, d), raw(d) if stream is None else _stream(stream))
    if status != 0:
        raise ElutqError(status, "elutq_mx4_gemm")


def elutq_mx4_gemm_grouped(x_codes, x_scales, w_codes, w_scales, offsets, Y, M: int, N: int, K: int, E: int, fmt: int, alpha=None, stream=None) -> None:
    """Rows offsets[e] .. offsets[e+1] of X [M, K] times W_e^T: W [E * N, K], offsets int32 [E + 1], alpha fp32 [E]."""
    where = "elutq_mx4_gemm_grouped"
    _, grouped, types, _, raw = _PRODUCTS or _products()
    d = _mx4_check(where, x_codes, x_scales, w_codes, w_scales, Y, M, N, K, E * N, fmt)
    status = grouped(x_codes.data_ptr(), x_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), _small(where, "offsets", offsets, _TORCH[0].int32, E + 1, d),
                     Y.data_ptr(), types.get(Y.dtype, -1), M, N, K, E, fmt, 0 if alpha is None else _small(where, "alpha", alpha, _TORCH[0].float32, E, d),
                     raw(d) if stream is None else _stream(stream))
    if status != 0:
        raise ElutqError(status, where)


def elutq_mx4_test_wait_expiry(x_codes, x_scales, w_codes, w_scales, Y, M: int, N: int, K: int, fmt: int, wait_limit: int, stream=None) -> None:
    where = "elutq_mx4_test_wait_expiry"
    types = _products()[2]
    _mx4_check(where, x_codes, x_scales, w_codes, w_scales, Y, M, N, K, N, fmt)
    _check(lib().elutq_mx4_test_wait_expiry(x_codes.data_ptr(), x_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), Y.data_ptr(),
                                            types.get(Y.dtype, -1), M, N, K, fmt, wait_limit, _stream(stream)), where)


def elutq_device_status(stream=None) -> int:
    """0 unless a kernel gave up on a bounded wait (synchronises the stream)."""
    out = c_int(0)
    _check(lib().elutq_device_status(_stream(stream), ctypes.byref(out)), "elutq_device_status")
    return out.value


def _call_array(calls):
    """calls: sequence of (X, packed, Y, N, K[, flags]) with tensors or raw addresses -> ctypes array."""
    arr = (GemvCall * len(calls))()
    for i, c in enumerate(calls):
        X, packed, Y, N, K = c[:5]
        flags = c[5] if len(c) > 5 else 0
        arr[i] = GemvCall(X if isinstance(X, int) else _ptr(X), packed if isinstance(packed, int) else _ptr(packed),
                          Y if isinstance(Y, int) else _ptr(Y), N, K, flags)
    return arr


def elutq_chain_plan_bytes(calls) -> int:
    out = c_size_t(0)
    _check(lib().elutq_chain_plan_bytes(_call_array(calls), len(calls), ctypes.byref(out)), "elutq_chain_plan_bytes")
    return out.value


def elutq_chain_plan(calls, plan=None, stream=None):
    """Writes the plan of a list of M = 1 calls into a device buffer (allocated here when not given); returns it."""
    import torch
    if plan is None:
        plan = torch.empty(elutq_chain_plan_bytes(calls), dtype=torch.uint8, device="cuda")
    _check(lib().elutq_chain_plan(_call_array(calls), len(calls), _ptr(plan), plan.numel() * plan.element_size(),
                                  _stream(stream)), "elutq_chain_plan")
    return plan


def elutq_chain_run(plan, n_calls: int, stream=None) -> None:
    _check(lib().elutq_chain_run(_ptr(plan), n_calls, _stream(stream)), "elutq_chain_run")


def elutq_chain_run_opts(plan, n_calls: int, wait_limit: int = 0, stream=None) -> None:
    _check(lib().elutq_chain_run_opts(_ptr(plan), n_calls, wait_limit, _stream(stream)), "elutq_chain_run_opts")


def elutq_chain_run_host(plan, n_calls: int, x_dev, x_host, y_dev=None, y_host=None, stream=None) -> None:
    """x_host -> x_dev, the plan's launches, y_dev -> y_host, all on `stream` (whole tensors are copied; a pair that
    is None is not copied: e.g. when the plan's Y pointers name pinned host memory themselves)."""
    xb = 0 if x_host is None else x_host.numel() * x_host.element_size()
    yb = 0 if y_host is None else y_host.numel() * y_host.element_size()
    _check(lib().elutq_chain_run_host(_ptr(plan), n_calls, _ptr(x_dev), _ptr(x_host), xb, _ptr(y_dev), _ptr(y_host), yb,
                                      _stream(stream)), "elutq_chain_run_host")


def elutq_chain_status(plan, stream=None) -> int:
    out = c_int(0)
    _check(lib().elutq_chain_status(_ptr(plan), _stream(stream), ctypes.byref(out)), "elutq_chain_status")
    return out.value


def elutq_chain_forget(plan) -> None:
    _check(lib().elutq_chain_forget(_ptr(plan)), "elutq_chain_forget")


def elutq_chain_shares(N: int, K: int, n_ctas_max: int, cta_first: int = 0, independent: bool = True):
    """(shares, partition): shares[cta] = (first row block, end row block, first chunk, chunks, chunk group);
    partition = (chunks per CTA, row ranges, chunk groups, CTAs with a share).  Host logic only."""
    raw = (c_int * (4 * n_ctas_max))()
    part = (c_int * 4)()
    _check(lib().elutq_chain_shares(N, K, n_ctas_max, cta_first, 1 if independent else 0, raw, part), "elutq_chain_shares")
    shares = [(raw[4 * i], raw[4 * i + 1], raw[4 * i + 2], raw[4 * i + 3] & 0xffff, raw[4 * i + 3] >> 16) for i in range(n_ctas_max)]
    return shares, tuple(part)


def elutq_reserve(M: int, N: int, K: int, stream=None) -> None:
    _check(lib().elutq_reserve(M, N, K, _stream(stream)), "elutq_reserve")


def elutq_scratch_address(kind: int, stream=None):
    """(address or None, bytes) of a library-owned scratch buffer of the stream."""
    ptr, nb = c_void_p(0), c_size_t(0)
    _check(lib().elutq_scratch_address(_stream(stream), kind, ctypes.byref(ptr), ctypes.byref(nb)), "elutq_scratch_address")
    return ptr.value, nb.value


def elutq_test_wait_expiry(X, packed, Y, M: int, N: int, K: int, wait_limit: int, stream=None) -> None:
    _check(lib().elutq_test_wait_expiry(_ptr(X), _ptr(packed), _ptr(Y), M, N, K, wait_limit, _stream(stream)),
           "elutq_test_wait_expiry")
