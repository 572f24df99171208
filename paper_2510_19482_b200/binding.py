"""ctypes binding: one Python function per C entry point, same names, argument marshalling only."""

from __future__ import annotations

import ctypes
import os
import struct
from ctypes import c_char_p, c_double, c_float, c_int, c_longlong, c_size_t, c_uint, c_ulonglong, c_void_p

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
KV_16, KV_E4M3, KV_NVFP4 = 0, 1, 2
ROPE_PLAIN, ROPE_LINEAR, ROPE_BANDS = 0, 1, 2
ROPE_INTERLEAVED = 0x1
ATTN_ALL_KEYS = 0x1
ATTN_TEST_LOADS = 0x80000000


class GemvCall(ctypes.Structure):
    """elutq_gemv_call: one M = 1 call of a chain."""
    _fields_ = [("X", c_void_p), ("packed", c_void_p), ("Y", c_void_p), ("N", c_int), ("K", c_int), ("flags", c_uint)]


class KvCacheDesc(ctypes.Structure):
    """elutq_kv_cache."""
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("k_scales", c_void_p), ("v_scales", c_void_p), ("k_factor", c_void_p), ("v_factor", c_void_p),
                ("format", c_int), ("type", c_int), ("n_pages", c_int), ("heads", c_int), ("page_size", c_int), ("head_dim", c_int)]


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
    "elutq_kv_bytes": (c_int, [c_int, c_int, c_int, c_int, c_int, ctypes.POINTER(c_size_t), ctypes.POINTER(c_size_t)]),
    "elutq_rope_table": (c_int, [c_void_p, c_int, c_int, c_double, c_int, c_double, c_double, c_double, c_double, c_double, c_void_p]),
    "elutq_kv_write": (c_int, [c_void_p, c_void_p, c_longlong, c_void_p, c_longlong, c_int, c_void_p, c_longlong, c_void_p, c_longlong, c_void_p, c_longlong, c_int,
                               c_void_p, c_void_p, c_void_p, c_int, c_int, c_uint, c_void_p]),
    "elutq_kv_read": (c_int, [c_void_p, c_void_p, c_longlong, c_int, c_void_p, c_void_p, c_int, c_int, c_void_p, c_longlong, c_void_p, c_longlong, c_void_p]),
    "elutq_attn_decode_workspace_bytes": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_void_p]),
    "elutq_attn_decode": (c_int, [c_void_p, c_void_p, c_longlong, c_void_p, c_longlong, c_void_p, c_longlong, c_int, c_void_p, c_int, c_int, c_int, c_float,
                                  c_void_p, c_size_t, c_void_p]),
    "elutq_attn_prefill": (c_int, [c_void_p, c_longlong, c_void_p, c_longlong, c_void_p, c_longlong, c_void_p, c_longlong, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_int, c_float, c_uint,
                                   c_void_p]),
    "elutq_attn_test_wait_expiry": (c_int, [c_void_p, c_longlong, c_void_p, c_longlong, c_void_p, c_longlong, c_void_p, c_longlong, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_int, c_float, c_uint,
                                            c_uint, c_void_p]),
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


_DESC = struct.Struct("6Q6i")       # elutq_kv_cache


class KvCache:
    """A paged cache: k, v [n_pages, heads, page_size, row] (KV_16: values of `dtype`; KV_E4M3: bytes; KV_NVFP4: head_dim / 2 bytes of codes, with
    scales [n_pages, heads, page_size, head_dim / 16] of bytes), all dense; factors fp32 [heads] or None.  `dtype`: of queries, keys, values and results."""

    __slots__ = ("desc", "device", "dtype", "heads", "head_dim", "tensors")

    def __init__(self, fmt: int, dtype, k, v, k_scales=None, v_scales=None, k_factor=None, v_factor=None):
        torch, types, _, _ = _TORCH or _torch()
        d, shape, kind = k.get_device(), k.shape, types.get(dtype, TYPE_F32)
        if (kind == TYPE_F32 or not 0 <= fmt <= 2 or len(shape) != 4 or d < 0 or v.shape != shape or v.get_device() != d or not k.is_contiguous() or not v.is_contiguous() or
                (k.dtype is not dtype or v.dtype is not dtype if fmt == 0 else k.element_size() != 1 or v.element_size() != 1)):
            _refuse("KvCache", "a format, torch.float16 or torch.bfloat16, and k, v of one shape [n_pages, heads, page_size, row], of that type or of bytes, wanted", k, v)
        pages, heads, page, dim = shape
        ks = vs = kf = vf = 0
        if fmt == KV_NVFP4:
            dim *= 2
            n = pages * heads * page * (dim // 16)
            for t in (k_scales, v_scales):
                if t is None or t.nbytes != n or t.element_size() != 1 or not t.is_contiguous() or t.get_device() != d:
                    _refuse("KvCache", f"scales: {n} bytes wanted", t)
            ks, vs = k_scales.data_ptr(), v_scales.data_ptr()
        if k_factor is not None:
            kf = _small("KvCache", "k_factor", k_factor, torch.float32, heads, d)
        if v_factor is not None:
            vf = _small("KvCache", "v_factor", v_factor, torch.float32, heads, d)
        self.desc = _DESC.pack(k.data_ptr(), v.data_ptr(), ks, vs, kf, vf, fmt, kind, pages, heads, page, dim)
        self.device, self.dtype, self.heads, self.head_dim = d, dtype, heads, dim
        self.tensors = (k, v, k_scales, v_scales, k_factor, v_factor)      # (they live as long as the descriptor names them)


def elutq_kv_bytes(fmt: int, n_pages: int, heads: int, page_size: int, head_dim: int):
    """(bytes of k, as of v; bytes of its scales)."""
    data, scales = c_size_t(0), c_size_t(0)
    _check(lib().elutq_kv_bytes(fmt, n_pages, heads, page_size, head_dim, ctypes.byref(data), ctypes.byref(scales)), "elutq_kv_bytes")
    return data.value, scales.value


def elutq_rope_table(n_pos: int, rot_dim: int, theta: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                     original: float = 8192.0, magnitude: float = 1.0, table=None, stream=None):
    """Cosines and sines of positions, fp32 [n_pos, rot_dim] (allocated here when not given; give one with a stream that is not torch's current one)."""
    if table is None and stream is not None:
        _refuse("elutq_rope_table", "a stream of one's own needs a table of its own")
    torch, _, current, _ = _torch()
    d = current()
    if table is None:
        table = torch.empty((n_pos, rot_dim), device=f"cuda:{d}")
    _check(lib().elutq_rope_table(_small("elutq_rope_table", "table", table, torch.float32, n_pos * rot_dim, d), n_pos, rot_dim, theta, scaling, factor, low, high,
                                  original, magnitude, _stream(stream)), "elutq_rope_table")
    return table


_ATTENTION = None


def _attention():
    """What a call of these entries needs, looked up once: torch, the current device, a device's current stream, and the C functions."""
    global _ATTENTION
    if _ATTENTION is None:
        torch, _, current, raw = _torch()
        L = lib()
        _ATTENTION = (torch, torch.int32, torch.float32, current, raw, L.elutq_kv_write, L.elutq_kv_read, L.elutq_attn_decode, L.elutq_attn_decode_workspace_bytes)
    return _ATTENTION


def _rows(where: str, name: str, t, n: int, D: int, dtype, device: int, rows: int) -> int:
    """Distance between the tokens of [rows, n, D] with heads side by side, in elements."""
    stride = t.stride()
    if t.shape != (rows, n, D) or stride[2] != 1 or (stride[1] != D and n > 1) or t.dtype is not dtype or t.get_device() != device:
        _refuse(where, f"{name}: {rows} tokens of {n} heads of {D} values of {dtype}, the heads of a token side by side, wanted", t)
    return stride[0] if rows > 1 else n * D


def _pages(where: str, table, device: int):
    """(sequences, pages, distance between the rows) of a table of pages int32 [B, pages]."""
    B, pages = table.shape if table.dim() == 2 else (0, 0)
    if B < 1 or table.dtype is not _TORCH[0].int32 or table.get_device() != device or (pages > 1 and table.stride(1) != 1):
        _refuse(where, "table: int32, a row of pages for each sequence wanted", table)
    return B, pages, table.stride(0) if B > 1 else pages


def elutq_kv_write(cache: KvCache, k, v, slots, q=None, q_out=None, positions=None, rope=None, flags: int = 0, k_out=None, stream=None) -> None:
    """k, v [tokens, heads, head_dim] into the cache, q and k rotated; slots, positions int32 [tokens], rope fp32 [n_pos, rot_dim].
    q [tokens, query heads, head_dim] -> q_out; the rotated keys -> k_out, if given."""
    where = "elutq_kv_write"
    _, int32, float32, current, raw, write, _, _, _ = _ATTENTION or _attention()
    d, H, D, dtype, rows = cache.device, cache.heads, cache.head_dim, cache.dtype, k.shape[0]
    if d != current() or (q is None) != (q_out is None) or (rope is not None and (positions is None or rope.dim() != 2)):
        _refuse(where, "q with q_out, and rope [n_pos, rot_dim] with positions wanted", k, q, q_out, rope, positions)
    ldk, ldv = _rows(where, "k", k, H, D, dtype, d, rows), _rows(where, "v", v, H, D, dtype, d, rows)
    n = ldq = ldqo = ldko = n_pos = rot = 0
    if q is not None:
        n = q.shape[1] if q.dim() == 3 else -1
        ldq, ldqo = _rows(where, "q", q, n, D, dtype, d, rows), _rows(where, "q_out", q_out, n, D, dtype, d, rows)
    if k_out is not None:
        ldko = _rows(where, "k_out", k_out, H, D, dtype, d, rows)
    if rope is not None:
        n_pos, rot = rope.shape
    status = write(cache.desc, 0 if q is None else q.data_ptr(), ldq, 0 if q is None else q_out.data_ptr(), ldqo, n, k.data_ptr(), ldk, 0 if k_out is None else k_out.data_ptr(), ldko,
                   v.data_ptr(), ldv, rows, _small(where, "slots", slots, int32, rows, d), _small(where, "positions", positions, int32, rows, d),
                   _small(where, "rope", rope, float32, n_pos * rot, d), n_pos, rot, flags, raw(d) if stream is None else _stream(stream))
    if status != 0:
        raise ElutqError(status, where)


def elutq_kv_read(cache: KvCache, table, first, cu, k_out, v_out, stream=None) -> None:
    """Tokens first[b] .. of every sequence to rows cu[b] .. cu[b+1] of k_out, v_out [rows, heads, head_dim]; table int32 [B, pages], first int32 [B] or None,
    cu int32 [B + 1]."""
    where = "elutq_kv_read"
    _, int32, _, current, raw, _, read, _, _ = _ATTENTION or _attention()
    d, H, D, dtype, rows = cache.device, cache.heads, cache.head_dim, cache.dtype, k_out.shape[0]
    if d != current():
        _refuse(where, f"a cache on the current device wanted, cuda:{d} given", k_out)
    ldk, ldv = _rows(where, "k_out", k_out, H, D, dtype, d, rows), _rows(where, "v_out", v_out, H, D, dtype, d, rows)
    B, pages, ld = _pages(where, table, d)
    status = read(cache.desc, table.data_ptr(), ld, pages, _small(where, "first", first, int32, B, d), _small(where, "cu", cu, int32, B + 1, d), B, rows,
                  k_out.data_ptr(), ldk, v_out.data_ptr(), ldv, raw(d) if stream is None else _stream(stream))
    if status != 0:
        raise ElutqError(status, where)


def elutq_attn_decode_workspace_bytes(cache: KvCache, pages: int, B: int, new_tokens: int, n_q_heads: int) -> int:
    out = c_size_t(0)
    _check(lib().elutq_attn_decode_workspace_bytes(cache.desc, pages, B, new_tokens, n_q_heads, ctypes.addressof(out)), "elutq_attn_decode_workspace_bytes")
    return out.value


def elutq_attn_decode(cache: KvCache, q, out, table, lens, new_tokens: int = 1, scale=None, workspace=None, stream=None) -> None:
    """out = attention of q [B * new_tokens, query heads, head_dim], the last tokens of the sequences, over the cache; table int32 [B, pages], lens int32 [B].
    scale None: head_dim ** -0.5.  workspace None: taken from torch's allocator, if one is needed (give one with a stream that is not torch's current one)."""
    where = "elutq_attn_decode"
    torch, int32, _, current, raw, _, _, decode, size = _ATTENTION or _attention()
    d, D, dtype = cache.device, cache.head_dim, cache.dtype
    if d != current() or q.dim() != 3:
        _refuse(where, f"a cache on the current device (cuda:{d} given) and q [tokens, heads, head_dim] wanted", q)
    B, pages, ld = _pages(where, table, d)
    n, rows = q.shape[1], B * new_tokens
    ldq, ldo = _rows(where, "q", q, n, D, dtype, d, rows), _rows(where, "out", out, n, D, dtype, d, rows)
    address = nbytes = 0
    if workspace is None:
        need = c_size_t(0)
        status = size(cache.desc, pages, B, new_tokens, n, ctypes.byref(need))
        if status != 0:
            raise ElutqError(status, where)
        nbytes = need.value
        if nbytes != 0:
            if stream is not None:
                _refuse(where, f"a stream of one's own needs a workspace of its own: {nbytes} bytes")
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
            address = workspace.data_ptr()
    elif not workspace.is_contiguous() or workspace.get_device() != d:
        _refuse(where, "workspace wanted", workspace)
    else:
        address, nbytes = workspace.data_ptr(), workspace.nbytes
    status = decode(cache.desc, q.data_ptr(), ldq, out.data_ptr(), ldo, table.data_ptr(), ld, pages, _small(where, "lens", lens, int32, B, d), B, new_tokens, n,
                    D ** -0.5 if scale is None else scale, address, nbytes, raw(d) if stream is None else _stream(stream))
    if status != 0:
        raise ElutqError(status, where)


def _prefill(where: str, q, k, v, out, cu_q, cu_k, max_q, scale, causal, stream, *more) -> None:
    torch, types, current, raw = _torch()
    d, dtype = q.get_device(), q.dtype
    if q.dim() != 3 or k.dim() != 3 or d < 0 or d != current():
        _refuse(where, "q, k [tokens, heads, head_dim] wanted", q, k)
    (rows, n, D), (keys, H, _) = q.shape, k.shape
    B = cu_q.numel() - 1
    _check(getattr(lib(), where)(q.data_ptr(), _rows(where, "q", q, n, D, dtype, d, rows), k.data_ptr(), _rows(where, "k", k, H, D, dtype, d, keys), v.data_ptr(), _rows(where, "v", v, H, D, dtype, d, keys),
                                 out.data_ptr(), _rows(where, "out", out, n, D, dtype, d, rows), types.get(dtype, -1), _small(where, "cu_q", cu_q, torch.int32, B + 1, d),
                                 _small(where, "cu_k", cu_k, torch.int32, B + 1, d), B, max_q, rows, keys, n, H, D, D ** -0.5 if scale is None else scale,
                                 0 if causal else ATTN_ALL_KEYS, *more, raw(d) if stream is None else _stream(stream)), where)


def elutq_attn_prefill(q, k, v, out, cu_q, cu_k, max_q: int, scale=None, causal: bool = True, stream=None) -> None:
    """out = attention of prompts one behind the other: q, out fp16 or bf16 [total_q, query heads, head_dim], k, v [total_k, heads, head_dim],
    cu_q, cu_k int32 [B + 1]; scale None: head_dim ** -0.5."""
    _prefill("elutq_attn_prefill", q, k, v, out, cu_q, cu_k, max_q, scale, causal, stream)


def elutq_attn_test_wait_expiry(q, k, v, out, cu_q, cu_k, max_q: int, wait_limit: int, scale=None, causal: bool = True, stream=None) -> None:
    _prefill("elutq_attn_test_wait_expiry", q, k, v, out, cu_q, cu_k, max_q, scale, causal, stream, wait_limit)


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
