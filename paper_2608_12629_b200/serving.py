"""Binding of the serving operators (include/cake_serving.h): argument marshalling only.

Each function has the name of the C entry point it calls; PyTorch supplies device memory and the stream.  The checks and the call
are native (csrc/ext/serving_ext.cpp): a program makes these calls for kernels of a few microseconds.  As in `binding`, there is
no fallback: a missing library, a wrong type or a refused shape raises.

With `stream`, the outputs and the scratch that a call allocates belong to that stream, as if it were the current one.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import CakeError, _check

CAKE_KV_BF16, CAKE_KV_E4M3 = 0, 1
CAKE_RMSNORM_NONE = 1
CAKE_GEMM_OUT_FP32 = 1
CAKE_APPEND_INTERLEAVED = 1
CAKE_SERVING_HEADER_BYTES = 16640
CAKE_GEMM_FP8_MOST_WORKSPACE_BYTES = 19415296

SERVING_EXPORTS = [
    "cake_rmsnorm_quant", "cake_gemm_fp8_workspace_bytes", "cake_gemm_fp8", "cake_kv_append",
    "cake_paged_decode_workspace_bytes", "cake_paged_decode",
]

_E4M3 = torch.float8_e4m3fn
_BF16 = torch.bfloat16


class _CacheStruct(ctypes.Structure):
    """struct cake_paged_cache"""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("num_pages", ctypes.c_longlong),
                ("k_page_stride", ctypes.c_longlong), ("k_token_stride", ctypes.c_longlong), ("k_head_stride", ctypes.c_longlong),
                ("v_page_stride", ctypes.c_longlong), ("v_token_stride", ctypes.c_longlong), ("v_head_stride", ctypes.c_longlong),
                ("page_size", ctypes.c_int), ("Hkv", ctypes.c_int), ("D", ctypes.c_int), ("type", ctypes.c_int)]


_lib = None


def _load() -> ctypes.CDLL:
    """The C entry points through ctypes (the workspace sizes; tests of the ABI itself)."""
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, ll, i, u, sz, f = ctypes.c_void_p, ctypes.c_longlong, ctypes.c_int, ctypes.c_uint, ctypes.c_size_t, ctypes.c_float
        cache = ctypes.POINTER(_CacheStruct)
        L.cake_rmsnorm_quant.argtypes = [vp, ll, vp, ll, vp, ll, i, f, i, vp, vp, vp, vp, vp, u]
        L.cake_gemm_fp8_workspace_bytes.argtypes = [ll, i, i, ctypes.POINTER(sz)]
        L.cake_gemm_fp8.argtypes = [vp, ll, vp, vp, ll, vp, ll, i, i, vp, ll, vp, sz, vp, u]
        L.cake_kv_append.argtypes = [cache, vp, ll, vp, ll, vp, ll, i, vp, vp, vp, vp, ll, i, ll, vp, sz, vp, u]
        L.cake_paged_decode_workspace_bytes.argtypes = [ll, i, i, i, ctypes.POINTER(sz)]
        L.cake_paged_decode.argtypes = [vp, ll, ll, cache, vp, ll, ll, i, vp, ll, ll, ll, i, f, i, vp, vp, vp, sz, vp]
        for name in SERVING_EXPORTS:
            getattr(L, name).restype = i
        _lib = L
    return _lib


_ext = None


def _native():
    global _ext
    if _ext is None:
        binding.lib()                       # the same library, loaded once; raises if it is missing
        try:
            from . import _serving
        except ImportError as e:
            raise RuntimeError("the serving operators' marshalling module cannot be loaded: build it with "
                               "`python -m paper_2608_12629_b200.build`; there is no fallback path") from e
        _ext = _serving
    return _ext


def _empty(shape, dtype, device, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _workspace(n, device, stream=None):
    if stream is not None:               # zeroed ahead of the call, and not handed out again before its kernels are done
        with torch.cuda.stream(stream):
            return _workspace(n, device)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    ws[:CAKE_SERVING_HEADER_BYTES].zero_()
    return ws


# ------------------------------------------------------------------------------------------------------- rmsnorm_quant
def cake_rmsnorm_quant(x, weight=None, residual=None, eps=1e-6, group=128, out_residual=None, out_y=None, out_q=None,
                       out_scale=None, want_q=True, want_y=False, want_residual=None, stream=None, flags=0):
    """Norm of x (+ residual), bf16 [T,H] -> (q e4m3 [T,H], scale fp32 [T,ceil(H/128)] or [T,1] for group 0, y bf16, s bf16).

    An output that is not asked for (want_q, want_y, want_residual; by default q, and s where there is a residual) comes back as
    None.  out_residual may be `residual` or `x` themselves.
    """
    if want_q and out_q is None:
        out_q = _empty(x.shape, _E4M3, x.device, stream)
    if out_q is not None and out_scale is None:
        out_scale = _empty((x.shape[0], 1 if group == 0 else -(-x.shape[1] // 128)), torch.float32, x.device, stream)
    if out_residual is None and (residual is not None if want_residual is None else want_residual):
        out_residual = _empty(x.shape, _BF16, x.device, stream)
    if want_y and out_y is None:
        out_y = _empty(x.shape, _BF16, x.device, stream)
    rc = (_ext or _native()).rmsnorm_quant(x, weight, residual, eps, group, out_residual, out_y, out_q, out_scale,
                                           None if stream is None else stream.cuda_stream, flags)
    if rc:
        raise CakeError(rc, "cake_rmsnorm_quant")
    return out_q, out_scale, out_y, out_residual


# ------------------------------------------------------------------------------------------------------------ gemm_fp8
def cake_gemm_fp8_workspace_bytes(M, N, K) -> int:
    out = ctypes.c_size_t(0)
    _check(_load().cake_gemm_fp8_workspace_bytes(M, N, K, ctypes.byref(out)), "cake_gemm_fp8_workspace_bytes")
    return int(out.value)


def alloc_gemm_workspace(M, N, K, device) -> torch.Tensor:
    """A workspace for cake_gemm_fp8 of this size, its header zeroed; with M None, of any number of rows (fewer may need more)."""
    return _workspace(CAKE_GEMM_FP8_MOST_WORKSPACE_BYTES if M is None else cake_gemm_fp8_workspace_bytes(M, N, K), device)


def cake_gemm_fp8(X, x_scale, W, w_scale, out=None, out_dtype=_BF16, ws=None, stream=None):
    """X e4m3 [M,K] with scales fp32 [M,ceil(K/128)], W e4m3 [N,K] with scales fp32 [ceil(N/128),ceil(K/128)] -> X W^T, [M,N]
    in bf16 or fp32 (the type of `out` where it is given)."""
    if out is None:
        if out_dtype not in (_BF16, torch.float32):
            raise TypeError("out_dtype must be torch.bfloat16 or torch.float32")
        out = _empty((X.shape[0], W.shape[0]), out_dtype, X.device, stream)
    if ws is None:
        ws = _workspace(cake_gemm_fp8_workspace_bytes(X.shape[0], W.shape[0], X.shape[1]), X.device, stream)
    rc = (_ext or _native()).gemm_fp8(X, x_scale, W, w_scale, out, ws, None if stream is None else stream.cuda_stream)
    if rc:
        raise CakeError(rc, "cake_gemm_fp8")
    return out


# --------------------------------------------------------------------------------------------------------------- cache
class PagedCache:
    """A paged cache of keys and values: k and v [num_pages, page_size, Hkv, D], bf16 or e4m3, D contiguous, any other strides (a
    cache held head by head inside a page is passed as a transposed view).  k_scale, v_scale: fp32 [Hkv] or None (ones): an
    element x is held as x / scale.  Keeps the tensors alive; holds no copy."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in (_BF16, _E4M3):
            raise TypeError("k and v must be bf16 or e4m3 [num_pages, page_size, Hkv, D] of the same shape")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise TypeError("the last dimension of k and v must be contiguous")
        if not k.is_cuda:
            raise TypeError("the operators take CUDA tensors")
        pages, page, Hkv, D = k.shape
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if t is not None and (t.dtype != torch.float32 or t.shape != (Hkv,) or not t.is_contiguous()):
                raise TypeError(f"{name} must be a contiguous fp32 tensor of shape ({Hkv},)")
        for name, t in (("v", v), ("k_scale", k_scale), ("v_scale", v_scale)):
            if t is not None and t.device != k.device:
                raise ValueError(f"{name} is on {t.device}, not on {k.device}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.page_size, self.Hkv, self.D = pages, page, Hkv, D
        # (the stride of a dimension of one element says nothing, and may be any number)
        strides = [t.stride(i) if t.size(i) > 1 else 0 for t in (k, v) for i in range(3)]
        self._struct = _CacheStruct(k.data_ptr(), v.data_ptr(), None if k_scale is None else k_scale.data_ptr(),
                                    None if v_scale is None else v_scale.data_ptr(), pages, *strides, page, Hkv, D,
                                    CAKE_KV_E4M3 if k.dtype == _E4M3 else CAKE_KV_BF16)
        self._address = ctypes.addressof(self._struct)

    @property
    def device(self):
        return self.k.device


def alloc_append_workspace(device) -> torch.Tensor:
    """A workspace for cake_kv_append (its device status), zeroed."""
    return _workspace(CAKE_SERVING_HEADER_BYTES, device)


def cake_kv_append(cache, k, v, slots, positions=None, cos_sin=None, q=None, out_q=None, interleaved=False, ws=None, stream=None):
    """Writes k, v bf16 [T,Hkv,D] to `slots` (int64 [T], negative: skipped) of the cache; with cos_sin fp32 [positions, rot] (cosines,
    then sines) and positions int32 [T], keys and queries are rotated.  Returns the rotated queries (None without q); out_q may be q."""
    if q is None:
        out_q = None
    elif out_q is None:
        out_q = _empty(q.shape, _BF16, q.device, stream)
    if ws is None:
        ws = _workspace(CAKE_SERVING_HEADER_BYTES, k.device, stream)
    rc = (_ext or _native()).kv_append(cache._address, cache.k, k, v, slots, positions, cos_sin, q, out_q, interleaved, ws,
                                       None if stream is None else stream.cuda_stream)
    if rc:
        raise CakeError(rc, "cake_kv_append")
    return out_q


# -------------------------------------------------------------------------------------------------------- paged_decode
def cake_paged_decode_workspace_bytes(B, Hq, Hkv, D) -> int:
    out = ctypes.c_size_t(0)
    _check(_load().cake_paged_decode_workspace_bytes(B, Hq, Hkv, D, ctypes.byref(out)), "cake_paged_decode_workspace_bytes")
    return int(out.value)


def alloc_decode_workspace(B, Hq, Hkv, D, device) -> torch.Tensor:
    """A workspace for cake_paged_decode of this size, its header zeroed."""
    return _workspace(cake_paged_decode_workspace_bytes(B, Hq, Hkv, D), device)


def cake_paged_decode(q, cache, page_table, seq_lens, scale=None, window=0, out=None, out_lse=None, want_lse=False, ws=None,
                      stream=None):
    """Attention of one token per sequence: q bf16 [B,Hq,D] over the cache -> (out bf16 [B,Hq,D], lse fp32 [B,Hq] or None).

    page_table int32 [B,max_pages] and seq_lens int32 [B], or one per key-value head: [B,Hkv,max_pages] and [B,Hkv].
    scale defaults to 1/sqrt(D); window > 0 attends to the last `window` tokens.
    """
    if out is None:
        out = _empty(q.shape, _BF16, q.device, stream)
    if want_lse and out_lse is None:
        out_lse = _empty(q.shape[:2], torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(cake_paged_decode_workspace_bytes(q.shape[0], q.shape[1], cache.Hkv, cache.D), q.device, stream)
    rc = (_ext or _native()).paged_decode(q, cache._address, cache.k, page_table, seq_lens, cache.D ** -0.5 if scale is None else scale, window, out, out_lse,
                                          ws, None if stream is None else stream.cuda_stream)
    if rc:
        raise CakeError(rc, "cake_paged_decode")
    return out, out_lse
