"""Binding over the C ABI of ``libdeepgemm_hip.so`` (declared in ``include/deepgemm_hip.h``).

Argument marshalling only: every step of the path runs in the library's HIP kernels.  torch is
used for device memory and streams, nothing else.  The run-time calls go through ``_native.so``
(``csrc/binding_native.cpp``: the same checks and the call, in C++), tables and sizes through ctypes.
There is no CPU fallback: if either library has not been built, loading fails with an explicit error.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdeepgemm_hip.so")
NATIVE_PATH = os.path.join(_HERE, "_native.so")

DG_OK = 0
STATUS_NAMES = ("DG_OK", "DG_ERR_NULL", "DG_ERR_SHAPE", "DG_ERR_RANGE", "DG_ERR_BUFFER",
                "DG_ERR_UNSUPPORTED", "DG_ERR_HIP")
DG_LUT_I8, DG_LUT_I16, DG_LUT_F32 = 0, 1, 2
DG_KERNEL_AUTO, DG_KERNEL_PERM, DG_KERNEL_LDS, DG_KERNEL_MFMA_I8, DG_KERNEL_SMALLN, DG_KERNEL_LUT65K = 0, 1, 2, 3, 4, 5
DG_KERNEL_ONEHOT_MFMA = 6
DG_KERNEL_ONEHOT_SMFMAC = 7
KERNELS = {"auto": DG_KERNEL_AUTO, "perm": DG_KERNEL_PERM, "lds": DG_KERNEL_LDS,
           "mfma_i8": DG_KERNEL_MFMA_I8, "smalln": DG_KERNEL_SMALLN, "lut65k": DG_KERNEL_LUT65K,
           "onehot_mfma": DG_KERNEL_ONEHOT_MFMA, "onehot_smfmac": DG_KERNEL_ONEHOT_SMFMAC}
ROUTE_MODES = {"softmax": 0, "softmax_all": 1, "sigmoid": 2}

# every symbol include/deepgemm_hip.h declares
EXPORTS = (
    "dg_status_string", "dg_last_error", "dg_build_lut", "dg_build_lut_bits", "dg_lut_bits", "dg_lut_entries",
    "dg_lut_entries_all", "dg_lut_destroy", "dg_build_lut_entries", "dg_build_lut_f32", "dg_lut_entries_f32",
    "dg_packed_activation_bytes", "dg_packed_weight_bytes", "dg_packed_bytes_bits", "dg_pack_weights",
    "dg_pack_activations", "dg_pack_codes_bits", "dg_quantize_pack_activations",
    "dg_gemm_lut", "dg_conv_out_dim", "dg_conv2d_lut", "dg_gemm_kernel_name", "dg_conv_kernel_name",
    "dg_conv2d_lut_codes", "dg_conv_codes_kernel_name", "dg_gemm_lut_codes", "dg_gemm_codes_kernel_name",
    "dg_launch_empty", "dg_dequantize", "dg_conv2d_lut_requant",
    "dg_static_work_bytes", "dg_conv2d_lut_codes_static",
    "dg_quantize_tokens", "dg_gemm_i8", "dg_linear_i8_work_bytes", "dg_linear_i8", "dg_cache_bytes", "dg_cache_write", "dg_cache_read",
    "dg_paged_attention_work_bytes", "dg_paged_attention",
    "dg_quantize_mx4", "dg_dequantize_mx4", "dg_gemm_mx4", "dg_linear_mx4_work_bytes", "dg_linear_mx4", "dg_route_tokens_work_bytes", "dg_route_tokens",
    "dg_experts_mx4_work_bytes", "dg_experts_mx4",
)


class ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "H", "W", "Cin", "Cout", "KH", "KW", "stride_h", "stride_w", "pad_h", "pad_w")]


class CacheDesc(ctypes.Structure):
    """A paged cache of quantised keys and values: its pages, their tokens, the heads, their channels, the bits of a code."""
    _fields_ = [(n, ctypes.c_int32) for n in ("pages", "page_size", "heads", "dim", "bits")]


class ExpertsDesc(ctypes.Structure):
    """Experts' weights in microscaled 4-bit floating point: how many, their sizes, where they lie (distances in bytes)."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("experts", "hidden", "inner", "reserved")]
                + [(n, ctypes.c_void_p) for n in ("up", "up_scales", "down", "down_scales")]
                + [(n, ctypes.c_int64) for n in ("up_row", "up_expert", "up_scales_row", "up_scales_expert",
                                                 "down_row", "down_expert", "down_scales_row", "down_scales_expert")])


class DgError(RuntimeError):
    def __init__(self, status: int, detail: str):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else f"status {status}"
        super().__init__(f"{name}: {detail}")


_lib = None


def lib() -> ctypes.CDLL:
    """Load the library (once).  Raises if it has not been built: there is no other path."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2304_09049_amd.build` "
                          "(hipcc, gfx950).  This package has no CPU fallback.")
    L = ctypes.CDLL(LIB_PATH)
    c_i64, c_vp, c_sz, c_int = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    L.dg_status_string.argtypes, L.dg_status_string.restype = [c_int], ctypes.c_char_p
    L.dg_last_error.argtypes, L.dg_last_error.restype = [], ctypes.c_char_p
    L.dg_build_lut.argtypes, L.dg_build_lut.restype = [c_vp, c_vp, c_int, ctypes.POINTER(c_vp)], c_int
    L.dg_lut_entries.argtypes, L.dg_lut_entries.restype = [c_vp, c_vp], c_int
    L.dg_build_lut_entries.argtypes, L.dg_build_lut_entries.restype = [c_vp, c_int, ctypes.POINTER(c_vp)], c_int
    L.dg_build_lut_f32.argtypes, L.dg_build_lut_f32.restype = [c_vp, c_vp, ctypes.POINTER(c_vp)], c_int
    L.dg_lut_entries_f32.argtypes, L.dg_lut_entries_f32.restype = [c_vp, c_vp], c_int
    L.dg_build_lut_bits.argtypes = [ctypes.c_int32, c_vp, c_vp, c_int, ctypes.POINTER(c_vp)]
    L.dg_build_lut_bits.restype = c_int
    L.dg_lut_bits.argtypes, L.dg_lut_bits.restype = [c_vp], ctypes.c_int32
    L.dg_lut_entries_all.argtypes, L.dg_lut_entries_all.restype = [c_vp, c_vp, ctypes.c_int32], c_int
    L.dg_packed_bytes_bits.argtypes, L.dg_packed_bytes_bits.restype = [c_i64, c_i64, ctypes.c_int32], c_sz
    L.dg_pack_codes_bits.argtypes = [c_vp, c_i64, c_i64, ctypes.c_int32, c_vp, c_sz, c_vp]
    L.dg_pack_codes_bits.restype = c_int
    L.dg_lut_destroy.argtypes, L.dg_lut_destroy.restype = [c_vp], None
    L.dg_packed_activation_bytes.argtypes, L.dg_packed_activation_bytes.restype = [c_i64, c_i64], c_sz
    L.dg_packed_weight_bytes.argtypes, L.dg_packed_weight_bytes.restype = [c_i64, c_i64], c_sz
    for f in (L.dg_pack_weights, L.dg_pack_activations):
        f.argtypes, f.restype = [c_vp, c_i64, c_i64, c_vp, c_sz, c_vp], c_int
    L.dg_quantize_pack_activations.argtypes = [c_vp, c_i64, c_i64, ctypes.c_float, ctypes.c_float, ctypes.c_int32,
                                               c_vp, c_sz, c_vp]
    L.dg_quantize_pack_activations.restype = c_int
    L.dg_gemm_lut.argtypes = [c_vp, c_vp, c_vp, c_i64, c_i64, c_i64, c_vp, c_i64, c_i64, c_vp, c_vp, c_int, c_vp]
    L.dg_gemm_lut.restype = c_int
    L.dg_conv_out_dim.argtypes, L.dg_conv_out_dim.restype = [c_i64] * 4, c_i64
    L.dg_conv2d_lut.argtypes = [c_vp, c_vp, c_vp, ctypes.POINTER(ConvDesc), c_vp, c_vp, c_vp, c_int, c_vp]
    L.dg_conv2d_lut.restype = c_int
    L.dg_gemm_kernel_name.argtypes, L.dg_gemm_kernel_name.restype = [c_vp, c_i64, c_i64, c_i64, c_int], ctypes.c_char_p
    L.dg_conv_kernel_name.argtypes = [c_vp, ctypes.POINTER(ConvDesc), c_int]
    L.dg_conv_kernel_name.restype = ctypes.c_char_p
    L.dg_conv2d_lut_codes.argtypes = [c_vp, c_vp, c_vp, ctypes.POINTER(ConvDesc), c_vp, c_sz, c_vp, c_vp, c_vp, c_int, c_vp]
    L.dg_conv2d_lut_codes.restype = c_int
    L.dg_static_work_bytes.argtypes, L.dg_static_work_bytes.restype = [], c_sz
    L.dg_conv2d_lut_codes_static.argtypes = [c_vp, c_vp, c_vp, ctypes.POINTER(ConvDesc), c_vp, c_vp, c_vp, c_int, c_vp]
    L.dg_conv2d_lut_codes_static.restype = c_int
    L.dg_gemm_lut_codes.argtypes = [c_vp, c_vp, c_vp, c_i64, c_i64, c_i64, c_vp, c_sz, c_vp, c_i64, c_i64, c_vp, c_vp, c_int, c_vp]
    L.dg_gemm_lut_codes.restype = c_int
    L.dg_gemm_codes_kernel_name.argtypes = [c_vp, c_i64, c_i64, c_i64, c_int]
    L.dg_gemm_codes_kernel_name.restype = ctypes.c_char_p
    L.dg_conv_codes_kernel_name.argtypes = [c_vp, ctypes.POINTER(ConvDesc), c_int]
    L.dg_conv_codes_kernel_name.restype = ctypes.c_char_p
    L.dg_launch_empty.argtypes, L.dg_launch_empty.restype = [c_i64, c_int, c_vp], c_int
    L.dg_dequantize.argtypes, L.dg_dequantize.restype = [c_vp, c_i64, c_i64, c_vp, c_vp, c_vp], c_int
    L.dg_conv2d_lut_requant.argtypes = [c_vp, c_vp, c_vp, ctypes.POINTER(ConvDesc), c_vp, ctypes.c_float, ctypes.c_float,
                                        ctypes.c_int32, c_vp, ctypes.c_size_t, c_int, c_vp]
    L.dg_conv2d_lut_requant.restype = c_int
    c_f, c_i32, desc = ctypes.c_float, ctypes.c_int32, ctypes.POINTER(CacheDesc)
    L.dg_quantize_tokens.argtypes, L.dg_quantize_tokens.restype = [c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_i64, c_vp, c_vp], c_int
    L.dg_gemm_i8.argtypes = [c_vp, c_i64, c_vp, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp, c_int, c_i64, c_vp]
    L.dg_gemm_i8.restype = c_int
    L.dg_linear_i8_work_bytes.argtypes, L.dg_linear_i8_work_bytes.restype = [c_i64, c_i64], c_sz
    L.dg_linear_i8.argtypes = [c_vp, c_i64, c_vp, c_int, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp, c_vp, c_sz, c_vp, c_int, c_i64, c_vp]
    L.dg_linear_i8.restype = c_int
    L.dg_cache_bytes.argtypes, L.dg_cache_bytes.restype = [desc], c_sz
    L.dg_cache_write.argtypes = [desc, c_vp, c_sz, c_vp, c_vp, c_int, c_i64, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp]
    L.dg_cache_write.restype = c_int
    L.dg_cache_read.argtypes, L.dg_cache_read.restype = [desc, c_vp, c_sz, c_vp, c_i64, c_vp, c_vp, c_int, c_vp], c_int
    L.dg_paged_attention_work_bytes.argtypes, L.dg_paged_attention_work_bytes.restype = [desc, c_i64, c_i64, c_i64, c_i64], c_sz
    L.dg_paged_attention.argtypes = [desc, c_vp, c_sz, c_vp, c_int, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp, c_vp, c_i64, c_i64, c_i64, c_i64,
                                     c_f, c_i32, c_vp, c_i64, c_i64, c_vp, c_sz, c_vp]
    L.dg_paged_attention.restype = c_int
    L.dg_quantize_mx4.argtypes, L.dg_quantize_mx4.restype = [c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_i64, c_vp, c_i64, c_vp], c_int
    L.dg_dequantize_mx4.argtypes, L.dg_dequantize_mx4.restype = [c_vp, c_i64, c_vp, c_i64, c_i64, c_i64, c_vp, c_int, c_i64, c_vp], c_int
    L.dg_gemm_mx4.argtypes = [c_vp, c_i64, c_vp, c_i64, c_vp, c_i64, c_vp, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp, c_int, c_i64, c_vp]
    L.dg_gemm_mx4.restype = c_int
    L.dg_linear_mx4_work_bytes.argtypes, L.dg_linear_mx4_work_bytes.restype = [c_i64, c_i64], c_sz
    L.dg_linear_mx4.argtypes = [c_vp, c_i64, c_vp, c_i64, c_vp, c_int, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp, c_sz, c_vp, c_int, c_i64, c_vp]
    L.dg_linear_mx4.restype = c_int
    L.dg_route_tokens_work_bytes.argtypes, L.dg_route_tokens_work_bytes.restype = [c_i64, c_i64], c_sz
    L.dg_route_tokens.argtypes = [c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_int, c_i64, c_i64, c_vp, c_i64, c_int, c_f, c_vp, c_vp, c_vp, c_sz, c_vp]
    L.dg_route_tokens.restype = c_int
    L.dg_experts_mx4_work_bytes.argtypes, L.dg_experts_mx4_work_bytes.restype = [c_i64] * 4, c_sz
    L.dg_experts_mx4.argtypes = [ctypes.POINTER(ExpertsDesc), c_vp, c_int, c_i64, c_i64, c_vp, c_vp, c_i64, c_vp, c_sz, c_vp, c_i64, c_vp]
    L.dg_experts_mx4.restype = c_int
    _lib = L
    return L


_native = None


def _load_native():
    """Load the native marshalling module (once).  Raises if it has not been built: there is no other path."""
    global _native
    lib()
    import torch  # noqa: F401  (the module uses torch's libraries)
    if not os.path.exists(NATIVE_PATH):
        raise ImportError(f"{NATIVE_PATH} is missing: build it with `python -m paper_2304_09049_amd.build`.")
    from . import _native as module
    module.use_desc(ConvDesc, CacheDesc)
    _native = module
    return module


def _check(status: int) -> None:
    if status != DG_OK:
        raise DgError(status, lib().dg_last_error().decode())


def _kernel(variant) -> int:
    return KERNELS[variant] if isinstance(variant, str) else int(variant)


def _stream_ptr(stream) -> ctypes.c_void_p:
    """hipStream_t of a torch stream (default: torch's current stream)."""
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


class Lut:
    """Owner of a ``dg_lut`` built by ``dg_build_lut``."""

    def __init__(self, levels_w: Sequence[int], levels_a: Sequence[int], entry: int = DG_LUT_I8, bits: int = 2,
                 entries: Optional[Sequence[int]] = None):
        self._h = None
        self._address = 0                             # the handle as a number, for the native module
        self.bits = bits
        self.is_f32 = entry == DG_LUT_F32
        handle = ctypes.c_void_p(0)
        if entries is not None:                       # a table given as such (any 16 integers)
            arr = (ctypes.c_int16 * 16)(*[int(v) for v in entries])
            _check(lib().dg_build_lut_entries(arr, int(entry), ctypes.byref(handle)))
            self._h, self._address = handle, handle.value
            return
        if self.is_f32:                               # binary32 products of floating-point levels
            lwf = (ctypes.c_float * 4)(*[float(v) for v in levels_w])
            laf = (ctypes.c_float * 4)(*[float(v) for v in levels_a])
            _check(lib().dg_build_lut_f32(lwf, laf, ctypes.byref(handle)))
            self._h, self._address = handle, handle.value
            return
        nlev = 1 << bits
        if len(levels_w) != nlev or len(levels_a) != nlev:
            raise ValueError(f"{bits}-bit codes need {nlev} levels per side")
        lw = (ctypes.c_int8 * nlev)(*[int(v) for v in levels_w])
        la = (ctypes.c_int8 * nlev)(*[int(v) for v in levels_a])
        if bits == 2:
            _check(lib().dg_build_lut(lw, la, int(entry), ctypes.byref(handle)))
        else:
            _check(lib().dg_build_lut_bits(bits, lw, la, int(entry), ctypes.byref(handle)))
        self._h, self._address = handle, handle.value

    @property
    def handle(self) -> ctypes.c_void_p:
        return self._h

    def entries(self):
        if self.is_f32:
            outf = (ctypes.c_float * 16)()
            _check(lib().dg_lut_entries_f32(self._h, outf))
            return list(outf)
        count = 1 << (2 * self.bits)
        out = (ctypes.c_int16 * count)()
        if self.bits == 2:
            _check(lib().dg_lut_entries(self._h, out))
        else:
            _check(lib().dg_lut_entries_all(self._h, out, count))
        return list(out)

    def __del__(self):
        if getattr(self, "_h", None) is not None and _lib is not None:
            _lib.dg_lut_destroy(self._h)
            self._h, self._address = None, 0


def dg_build_lut(levels_w, levels_a, entry: int = DG_LUT_I8) -> Lut:
    return Lut(levels_w, levels_a, entry)


def dg_build_lut_entries(entries, entry: int = DG_LUT_I16) -> Lut:
    return Lut((), (), entry, entries=entries)


def dg_build_lut_f32(levels_w, levels_a) -> Lut:
    return Lut(levels_w, levels_a, DG_LUT_F32)


def dg_build_lut_bits(bits: int, levels_w, levels_a, entry: int = DG_LUT_I8) -> Lut:
    return Lut(levels_w, levels_a, entry, bits=bits)


def dg_packed_bytes_bits(rows: int, K: int, bits: int) -> int:
    return int(lib().dg_packed_bytes_bits(rows, K, bits))


def dg_pack_codes_bits(codes, rows: int, K: int, bits: int, out=None, stream=None):
    """codes: uint8 device tensor with rows*K elements of `bits`-bit codes -> packed uint8 tensor (weights or activations)."""
    if out is None:
        import torch
        out = torch.empty(dg_packed_bytes_bits(rows, K, bits), dtype=torch.uint8, device=codes.device)
    status = (_native or _load_native()).pack_codes_bits(codes, rows, K, bits, out, stream)
    if status:
        _check(status)
    return out


def dg_packed_activation_bytes(rows: int, K: int) -> int:
    return int(lib().dg_packed_activation_bytes(rows, K))


def dg_packed_weight_bytes(M: int, K: int) -> int:
    return int(lib().dg_packed_weight_bytes(M, K))


def dg_conv_out_dim(size: int, k: int, stride: int, pad: int) -> int:
    return int(lib().dg_conv_out_dim(size, k, stride, pad))


def dg_pack_weights(codes, M: int, K: int, out=None, stream=None):
    """codes: uint8 device tensor with M*K elements ([M][K], or [Cout][KH][KW][Cin]) -> packed uint8 tensor."""
    if out is None:
        import torch
        out = torch.empty(dg_packed_weight_bytes(M, K), dtype=torch.uint8, device=codes.device)
    status = (_native or _load_native()).pack_weights(codes, M, K, out, stream)
    if status:
        _check(status)
    return out


def dg_pack_activations(codes, N: int, K: int, out=None, stream=None):
    """codes: uint8 device tensor with N*K elements ([N][K], or NHWC with N = B*H*W, K = C) -> packed uint8 tensor."""
    if out is None:
        import torch
        out = torch.empty(dg_packed_activation_bytes(N, K), dtype=torch.uint8, device=codes.device)
    status = (_native or _load_native()).pack_activations(codes, N, K, out, stream)
    if status:
        _check(status)
    return out


def dg_quantize_pack_activations(x, N: int, K: int, scale: float, zero_point: float, lo: int, out=None, stream=None):
    """x: float32 device tensor with N*K elements -> packed 2-bit codes of clip(rint(scale*x + zero_point), lo, lo+3) - lo."""
    if out is None:
        import torch
        out = torch.empty(dg_packed_activation_bytes(N, K), dtype=torch.uint8, device=x.device)
    status = (_native or _load_native()).quantize_pack_activations(x, N, K, scale, zero_point, lo, out, stream)
    if status:
        _check(status)
    return out


def _empty(shape, lut: Lut, scale, device):
    import torch
    return torch.empty(shape, dtype=torch.float32 if scale is not None or lut.is_f32 else torch.int32, device=device)


def dg_gemm_lut(lut: Lut, Wp, Ap, M: int, N: int, K: int, out=None, scale=None, variant="auto",
                stream=None, strides: Optional[Sequence[int]] = None):
    """C[m][n] = sum_k LUT[4*Wc[m][k] + Ac[n][k]].  Returns int32 [M][N], or float32 when `scale` is given."""
    if out is None:
        out = _empty((M, N), lut, scale, Wp.device)
    scm, scn = (N, 1) if strides is None else strides
    status = (_native or _load_native()).gemm_lut(lut, lut.is_f32, Wp, Ap, M, N, K, out, scm, scn, scale,
                                                  _kernel(variant), stream)
    if status:
        _check(status)
    return out


def dg_gemm_lut_codes(lut: Lut, Wp, Ac, M: int, N: int, K: int, work=None, out=None, scale=None, variant="auto",
                      stream=None, strides: Optional[Sequence[int]] = None):
    """Packing stage + GEMM as one call, from codes one per byte (`Ac`: uint8 [N][K]).  `work` is the packed-activation
    buffer the library uses when it does not fuse the packing into the kernel (may be None)."""
    if out is None:
        out = _empty((M, N), lut, scale, Wp.device)
    scm, scn = (N, 1) if strides is None else strides
    status = (_native or _load_native()).gemm_lut_codes(lut, lut.is_f32, Wp, Ac, M, N, K, work, out, scm, scn, scale,
                                                        _kernel(variant), stream)
    if status:
        _check(status)
    return out


def dg_gemm_codes_kernel_name(lut: Lut, M: int, N: int, K: int, variant="auto") -> str:
    return lib().dg_gemm_codes_kernel_name(lut.handle, M, N, K, _kernel(variant)).decode()


def conv_desc(B, H, W, Cin, Cout, KH, KW, stride=(1, 1), pad=(0, 0)) -> ConvDesc:
    return ConvDesc(B, H, W, Cin, Cout, KH, KW, stride[0], stride[1], pad[0], pad[1])


def _conv_shape(desc: ConvDesc):
    OH = dg_conv_out_dim(desc.H, desc.KH, desc.stride_h, desc.pad_h)
    OW = dg_conv_out_dim(desc.W, desc.KW, desc.stride_w, desc.pad_w)
    return desc.B, max(OH, 0), max(OW, 0), desc.Cout


def dg_conv2d_lut(lut: Lut, Wp, Xp, desc: ConvDesc, out=None, scale=None, variant="auto", stream=None):
    """NHWC convolution by table lookup.  Returns [B][OH][OW][Cout], int32 or float32 (when `scale` is given)."""
    if out is None:
        out = _empty(_conv_shape(desc), lut, scale, Wp.device)
    status = (_native or _load_native()).conv2d_lut(lut, lut.is_f32, Wp, Xp, desc, out, scale, _kernel(variant), stream)
    if status:
        _check(status)
    return out


def dg_conv2d_lut_codes(lut: Lut, Wp, Xc, desc: ConvDesc, work=None, out=None, scale=None, variant="auto", stream=None):
    """Packing stage + NHWC convolution as one call, from codes one per byte (`Xc`: uint8 [B][H][W][Cin]).  `work` is
    the packed-activation buffer the library uses when it does not fuse the packing into the kernel (may be None)."""
    if out is None:
        out = _empty(_conv_shape(desc), lut, scale, Wp.device)
    status = (_native or _load_native()).conv2d_lut_codes(lut, lut.is_f32, Wp, Xc, desc, work, out, scale,
                                                          _kernel(variant), stream)
    if status:
        _check(status)
    return out


def dg_static_work_bytes() -> int:
    return int(lib().dg_static_work_bytes())


def dg_conv2d_lut_codes_static(lut: Lut, Wp, Xc, desc: ConvDesc, out, scale=None, variant="auto", stream=None):
    """dg_conv2d_lut_codes with the library's own staging buffer; `out` is required (the call allocates nothing)."""
    status = (_native or _load_native()).conv2d_lut_codes_static(lut, lut.is_f32, Wp, Xc, desc, out, scale,
                                                                 _kernel(variant), stream)
    if status:
        _check(status)
    return out


def dg_conv_codes_kernel_name(lut: Lut, desc: ConvDesc, variant="auto") -> str:
    return lib().dg_conv_codes_kernel_name(lut.handle, ctypes.byref(desc), _kernel(variant)).decode()


def dg_gemm_kernel_name(lut: Lut, M: int, N: int, K: int, variant="auto") -> str:
    return lib().dg_gemm_kernel_name(lut.handle, M, N, K, _kernel(variant)).decode()


def dg_conv_kernel_name(lut: Lut, desc: ConvDesc, variant="auto") -> str:
    return lib().dg_conv_kernel_name(lut.handle, ctypes.byref(desc), _kernel(variant)).decode()


def dg_launch_empty(blocks: int, threads: int, stream=None) -> None:
    """A launch that does nothing: the cost of a grid of that shape (measurement aid)."""
    _check(lib().dg_launch_empty(blocks, threads, _stream_ptr(stream)))


def dg_dequantize(acc, rows: int, C: int, scale, out=None, stream=None):
    """acc: int32 device tensor [rows][C]; scale: float32 [C] -> float32 [rows][C] = float(acc) * scale[c]."""
    if out is None:
        import torch
        out = torch.empty(acc.shape, dtype=torch.float32, device=acc.device)
    status = (_native or _load_native()).dequantize(acc, rows, C, scale, out, stream)
    if status:
        _check(status)
    return out


def dg_conv2d_lut_requant(lut: Lut, Wp, Xp, desc: ConvDesc, scale, q_scale: float, q_zero: float, lo: int, out=None,
                          variant="auto", stream=None):
    """One fused layer: table convolution, per-channel scale, re-quantisation and packing -> packed uint8 [B*OH*OW][Cout/4]."""
    if out is None:
        import torch
        B, OH, OW, Cout = _conv_shape(desc)
        out = torch.empty(dg_packed_activation_bytes(B * OH * OW, Cout), dtype=torch.uint8, device=Wp.device)
    status = (_native or _load_native()).conv2d_lut_requant(lut, Wp, Xp, desc, scale, q_scale, q_zero, lo, out,
                                                            _kernel(variant), stream)
    if status:
        _check(status)
    return out


# ---- a quantised decoder layer around the tables ----------------------------------------------------------------------------


def _new(shape, dtype: str, device, stream):
    """A tensor for a call on `stream` (None: the current one), from that stream's memory: what the call leaves behind there, or drops before it
    has run, is given to no other stream's work."""
    import torch
    dtype = getattr(torch, dtype) if isinstance(dtype, str) else dtype
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def dg_quantize_tokens(x, codes=None, scale=None, stream=None):
    """x: float32, float16 or bfloat16 device tensor [N][K] (rows may lie apart) -> (int8 codes [N][K], float32 scale [N]): scale =
    max|x| / 127 of the row.  The codes made here are rows of whole 16 bytes (a view), as the product reads them fastest."""
    if codes is None:
        codes = _new((x.shape[0], -(-x.shape[1] // 16) * 16), "int8", x.device, stream)[:, :x.shape[1]]
    if scale is None:
        scale = _new(x.shape[0], "float32", x.device, stream)
    status = (_native or _load_native()).quantize_tokens(x, codes, scale, stream)
    if status:
        _check(status)
    return codes, scale


def dg_gemm_i8(W, A, scale_m, scale_n, bias=None, out=None, dtype=None, stream=None):
    """W: int8 [M][K]; A: int8 [N][K] -> [N][M] of `dtype` (or out's; default float32): the exact sums times scale_m[m] times scale_n[n], plus
    the float32 bias[m] if one is given."""
    if out is None:
        out = _new((A.shape[0], W.shape[0]), dtype or "float32", W.device, stream)
    status = (_native or _load_native()).gemm_i8(W, A, scale_m, scale_n, bias, out, stream)
    if status:
        _check(status)
    return out


def dg_linear_i8_work_bytes(N: int, K: int) -> int:
    return int(lib().dg_linear_i8_work_bytes(N, K))


def dg_linear_i8(W, x, scale_m, bias=None, work=None, out=None, stream=None):
    """dg_quantize_tokens and dg_gemm_i8 as one call: x [N][K] -> [N][M] of x's dtype (or out's).  `work`: uint8, dg_linear_i8_work_bytes(N, K)."""
    if out is None:
        out = _new((x.shape[0], W.shape[0]), x.dtype, W.device, stream)
    if work is None:
        work = _new(dg_linear_i8_work_bytes(x.shape[0], x.shape[1]), "uint8", W.device, stream)
    status = (_native or _load_native()).linear_i8(W, x, scale_m, bias, work, out, stream)
    if status:
        _check(status)
    return out


def cache_desc(pages: int, page_size: int, heads: int, dim: int, bits: int = 8) -> CacheDesc:
    return CacheDesc(pages, page_size, heads, dim, bits)


def dg_cache_bytes(desc: CacheDesc) -> int:
    return int(lib().dg_cache_bytes(ctypes.byref(desc)))


def dg_cache_write(desc: CacheDesc, cache, k, v, slots, stream=None) -> None:
    """k, v: [T][heads][dim] device tensors (tokens and heads may lie apart), quantised into `slots` (int32 [T]) of `cache` (uint8)."""
    status = (_native or _load_native()).cache_write(desc, cache, k, v, slots, stream)
    if status:
        _check(status)


def dg_cache_read(desc: CacheDesc, cache, slots, k_out=None, v_out=None, dtype=None, stream=None):
    """The keys and values that `slots` hold, [T][heads][dim] each, of `dtype` (default float32) or the outputs' own."""
    if k_out is None and v_out is None:
        k_out, v_out = (_new((slots.numel(), desc.heads, desc.dim), dtype or "float32", cache.device, stream) for _ in range(2))
    status = (_native or _load_native()).cache_read(desc, cache, slots, k_out, v_out, stream)
    if status:
        _check(status)
    return k_out, v_out


def dg_paged_attention_work_bytes(desc: CacheDesc, B: int, Hq: int, max_q: int, max_ctx: int) -> int:
    return int(lib().dg_paged_attention_work_bytes(ctypes.byref(desc), B, Hq, max_q, max_ctx))


def dg_paged_attention(desc: CacheDesc, cache, q, q_start, ctx_len, table, max_q: int, max_ctx: int, scale: Optional[float] = None,
                       causal: bool = True, out=None, work=None, stream=None):
    """Attention of a batch's new tokens over the cache.  q: [T][Hq][dim] float16 or bfloat16; sequence b has the rows q_start[b] ...
    q_start[b + 1] - 1 (int32 [B + 1]) and ctx_len[b] tokens (int32 [B], the new ones included) in the pages of table[b] (int32 [B][width]).
    max_q: the most new tokens of a sequence; max_ctx: about the longest context.  scale: default dim ** -0.5.  `work`: uint8,
    dg_paged_attention_work_bytes(desc, B, Hq, max_q, max_ctx)."""
    if out is None:
        out = _new(q.shape, q.dtype, q.device, stream)
    if work is None:
        need = dg_paged_attention_work_bytes(desc, table.shape[0], q.shape[1], max_q, max_ctx)
        if need:
            work = _new(need, "uint8", q.device, stream)
    status = (_native or _load_native()).paged_attention(desc, cache, q, q_start, ctx_len, table, max_q, max_ctx,
                                                         desc.dim ** -0.5 if scale is None else scale, causal, out, work, stream)
    if status:
        _check(status)
    return out


# ---- layers in microscaled 4-bit floating point, and layers of experts --------------------------------------------------------


def dg_quantize_mx4(x, codes=None, scales=None, stream=None):
    """x: float32, float16 or bfloat16 device tensor [N][K] (rows may lie apart) -> (codes, scales): uint8 [N][16 * blocks], two codes a byte, and uint8
    [N][blocks], a power of two for each block of 32.  The rows made here are views: scales' of whole words of
    four bytes, long codes' of whole cache lines (products of rows that begin inside one take up to a fifth longer)."""
    blocks = -(-x.shape[1] // 32)
    if codes is None:
        codes = _new((x.shape[0], 16 * blocks if blocks <= 64 else -(-blocks // 8) * 128), "uint8", x.device, stream)[:, :16 * blocks]
    if scales is None:
        scales = _new((x.shape[0], -(-blocks // 4) * 4), "uint8", x.device, stream)[:, :blocks]
    status = (_native or _load_native()).quantize_mx4(x, codes, scales, stream)
    if status:
        _check(status)
    return codes, scales


def dg_dequantize_mx4(codes, scales, K: Optional[int] = None, out=None, dtype=None, stream=None):
    """The values [N][K] (K: all that the blocks hold, if it is not given) of codes and scales, of `dtype` (default float32) or out's."""
    if out is None:
        out = _new((codes.shape[0], 2 * codes.shape[1] if K is None else K), dtype or "float32", codes.device, stream)
    elif K is not None and out.shape[1] != K:
        raise ValueError(f"out must have {K} columns, got {out.shape[1]}")
    status = (_native or _load_native()).dequantize_mx4(codes, scales, out, stream)
    if status:
        _check(status)
    return out


def dg_gemm_mx4(W, W_scales, A, A_scales, bias=None, out=None, dtype=None, stream=None):
    """Product of two quantised matrices, W [M rows] and A [N rows] of as many blocks -> [N][M] of `dtype` (or out's; default float32), plus the float32 bias[m] if
    one is given."""
    if out is None:
        out = _new((A.shape[0], W.shape[0]), dtype or "float32", W.device, stream)
    status = (_native or _load_native()).gemm_mx4(W, W_scales, A, A_scales, bias, out, stream)
    if status:
        _check(status)
    return out


def dg_linear_mx4_work_bytes(N: int, K: int) -> int:
    return int(lib().dg_linear_mx4_work_bytes(N, K))


def dg_linear_mx4(W, W_scales, x, bias=None, work=None, out=None, stream=None):
    """dg_quantize_mx4 and dg_gemm_mx4 as one call: x [N][K] -> [N][M] of x's dtype (or out's).  `work`: uint8, dg_linear_mx4_work_bytes(N, K)."""
    if out is None:
        out = _new((x.shape[0], W.shape[0]), x.dtype, W.device, stream)
    if work is None:
        work = _new(dg_linear_mx4_work_bytes(x.shape[0], x.shape[1]), "uint8", W.device, stream)
    status = (_native or _load_native()).linear_mx4(W, W_scales, x, bias, work, out, stream)
    if status:
        _check(status)
    return out


def dg_route_tokens_work_bytes(T: int, E: int) -> int:
    return int(lib().dg_route_tokens_work_bytes(T, E))


def dg_route_tokens(x, R, top: int, mode="softmax", bias=None, factor: float = 1.0, ids=None, weights=None, work=None, stream=None):
    """A router R [E][K] (x's dtype or float32) on tokens x [T][K] -> (ids int32 [T][top], weights float32 [T][top]): the experts of the `top` largest logits
    ("softmax": weights over those taken, "softmax_all": over all) or sigmoids ("sigmoid": normalised over those taken), with the float32 bias[e] added to what they are
    chosen by; weights times `factor`.  `work`: uint8, dg_route_tokens_work_bytes(T, E)."""
    if ids is None:
        ids = _new((x.shape[0], top), "int32", x.device, stream)
    if weights is None:
        weights = _new((x.shape[0], top), "float32", x.device, stream)
    if work is None:
        work = _new(dg_route_tokens_work_bytes(x.shape[0], R.shape[0]), "uint8", x.device, stream)
    status = (_native or _load_native()).route_tokens(x, R, top, ROUTE_MODES[mode] if isinstance(mode, str) else int(mode), bias, factor, ids, weights, work, stream)
    if status:
        _check(status)
    return ids, weights


def dg_experts_mx4_work_bytes(T: int, top: int, hidden: int, inner: int) -> int:
    return int(lib().dg_experts_mx4_work_bytes(T, top, hidden, inner))


def dg_experts_mx4(up, up_scales, down, down_scales, x, ids, weights, work=None, out=None, stream=None):
    """The gated feed-forward of the experts that ids [T][top] (int32) name, added up with weights [T][top] (float32): x [T][hidden] float16 or bfloat16 -> the
    same.  up: quantised [experts][2 * inner] rows of `hidden` (the gates' first), down: [experts][hidden] rows of `inner`, as dg_quantize_mx4 makes rows.
    `work`: uint8, dg_experts_mx4_work_bytes(T, top, hidden, inner)."""
    if out is None:
        out = _new(x.shape, x.dtype, x.device, stream)
    if work is None:
        work = _new(dg_experts_mx4_work_bytes(x.shape[0], ids.shape[1], x.shape[1], up.shape[1] // 2), "uint8", x.device, stream)
    status = (_native or _load_native()).experts_mx4(up, up_scales, down, down_scales, x, ids, weights, work, out, stream)
    if status:
        _check(status)
    return out
