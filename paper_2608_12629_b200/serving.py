"""ctypes binding of the serving operators (include/cake_serving.h): argument marshalling only.

Each function has the name of the C entry point it calls; PyTorch supplies device memory and the stream.  As in `binding`,
there is no fallback: a missing library, a wrong type or a refused shape raises.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import binding
from .binding import CakeError, _check, _want

CAKE_KV_BF16, CAKE_KV_E4M3 = 0, 1
CAKE_RMSNORM_NONE = 1
CAKE_GEMM_OUT_FP32 = 1
CAKE_APPEND_INTERLEAVED = 1
CAKE_SERVING_HEADER_BYTES = 16640

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


def _p(t):
    return None if t is None else t.data_ptr()


def _call(fn, where, device, stream, *args):
    """fn(*args, stream handle) with the tensors' device current.  `args` holds a None where the handle goes last but flags."""
    index = device.index
    if index == torch.cuda.current_device():
        rc = fn(*args, *_tail(stream, index))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, *_tail(stream, index))
    if rc != 0:
        raise CakeError(rc, where)


def _tail(stream, index):
    return (stream.cuda_stream if stream is not None else torch.cuda.current_stream(index).cuda_stream,)


def _on(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")
    if device.type != "cuda":
        raise TypeError("the operators take CUDA tensors")


def _rows(t, dtype, name):
    """A matrix whose rows are contiguous; returns (rows, columns, stride between rows)."""
    if t.dtype != dtype or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise TypeError(f"{name} must be a {dtype} matrix with contiguous rows")
    n, c = t.shape
    return n, c, (t.stride(0) if n > 1 else c)


def _dense(t, dtype, shape, name):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    return t


def _buffer(ws, need, name):
    if ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise TypeError(f"{name} must be a contiguous uint8 tensor")
    return ws


def _workspace(n, device):
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
    T, H, x_stride = _rows(x, _BF16, "x")
    device = x.device
    r_stride = H
    if residual is not None:
        if residual.shape != x.shape:
            raise ValueError("residual must have x's shape")
        r_stride = _rows(residual, _BF16, "residual")[2]
    if weight is not None:
        _dense(weight, _BF16, (H,), "weight")
    if want_residual is None:
        want_residual = residual is not None
    n = 1 if group == 0 else -(-H // 128)
    if out_residual is None and want_residual:
        out_residual = torch.empty(T, H, dtype=_BF16, device=device)
    if out_y is None and want_y:
        out_y = torch.empty(T, H, dtype=_BF16, device=device)
    if out_q is None and want_q:
        out_q = torch.empty(T, H, dtype=_E4M3, device=device)
    if out_scale is None and out_q is not None:
        out_scale = torch.empty(T, n, dtype=torch.float32, device=device)
    if out_residual is not None:
        _dense(out_residual, _BF16, (T, H), "out_residual")
    if out_y is not None:
        _dense(out_y, _BF16, (T, H), "out_y")
    if out_q is not None:
        _dense(out_q, _E4M3, (T, H), "out_q")
        _dense(out_scale, torch.float32, (T, n), "out_scale")
    _on(device, weight=weight, residual=residual, out_residual=out_residual, out_y=out_y, out_q=out_q, out_scale=out_scale)
    L = _load()
    fn = L.cake_rmsnorm_quant
    _call(lambda *a: fn(*a, flags), "cake_rmsnorm_quant", device, stream, _p(x), x_stride, _p(residual), r_stride, _p(weight), T, H,
          eps, group, _p(out_residual), _p(out_y), _p(out_q), _p(out_scale))
    return out_q, out_scale, out_y, out_residual


# ------------------------------------------------------------------------------------------------------------ gemm_fp8
def cake_gemm_fp8_workspace_bytes(M, N, K) -> int:
    out = ctypes.c_size_t(0)
    _check(_load().cake_gemm_fp8_workspace_bytes(M, N, K, ctypes.byref(out)), "cake_gemm_fp8_workspace_bytes")
    return int(out.value)


def alloc_gemm_workspace(M, N, K, device) -> torch.Tensor:
    """A workspace for cake_gemm_fp8 of this size, its header zeroed."""
    return _workspace(cake_gemm_fp8_workspace_bytes(M, N, K), device)


def cake_gemm_fp8(X, x_scale, W, w_scale, out=None, out_dtype=_BF16, ws=None, stream=None):
    """X e4m3 [M,K] with scales fp32 [M,ceil(K/128)], W e4m3 [N,K] with scales fp32 [ceil(N/128),ceil(K/128)] -> X W^T, [M,N]
    in bf16 or fp32 (the type of `out` where it is given)."""
    M, K, x_stride = _rows(X, _E4M3, "X")
    N, Kw, w_stride = _rows(W, _E4M3, "W")
    if K != Kw:
        raise ValueError("X must be [M,K] and W [N,K]")
    device = X.device
    nk = -(-K // 128)
    _dense(x_scale, torch.float32, (M, nk), "x_scale")
    _dense(w_scale, torch.float32, (-(-N // 128), nk), "w_scale")
    if out is None:
        if out_dtype not in (_BF16, torch.float32):
            raise TypeError("out_dtype must be torch.bfloat16 or torch.float32")
        out = torch.empty(M, N, dtype=out_dtype, device=device)
    elif out.dtype not in (_BF16, torch.float32) or out.shape != (M, N):
        raise TypeError("out must be a bf16 or fp32 [M,N] matrix")
    out_stride = _rows(out, out.dtype, "out")[2]
    if ws is None:
        ws = alloc_gemm_workspace(M, N, K, device)
    _buffer(ws, 0, "ws")
    _on(device, W=W, x_scale=x_scale, w_scale=w_scale, out=out, ws=ws)
    fn = _load().cake_gemm_fp8
    flags = CAKE_GEMM_OUT_FP32 if out.dtype == torch.float32 else 0
    _call(lambda *a: fn(*a, flags), "cake_gemm_fp8", device, stream, _p(X), x_stride, _p(x_scale), _p(W), w_stride, _p(w_scale), M, N, K,
          _p(out), out_stride, _p(ws), ws.numel())
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
        pages, page, Hkv, D = k.shape
        for name, s in (("k_scale", k_scale), ("v_scale", v_scale)):
            if s is not None:
                _dense(s, torch.float32, (Hkv,), name)
        _on(k.device, v=v, k_scale=k_scale, v_scale=v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.page_size, self.Hkv, self.D = pages, page, Hkv, D
        self.device = k.device
        self._struct = _CacheStruct(_p(k), _p(v), _p(k_scale), _p(v_scale), pages, k.stride(0), k.stride(1), k.stride(2), v.stride(0),
                                    v.stride(1), v.stride(2), page, Hkv, D, CAKE_KV_E4M3 if k.dtype == _E4M3 else CAKE_KV_BF16)
        self._ref = ctypes.byref(self._struct)


def alloc_append_workspace(device) -> torch.Tensor:
    """A workspace for cake_kv_append (its device status), zeroed."""
    return _workspace(CAKE_SERVING_HEADER_BYTES, device)


def _heads(t, D, name):
    """[T, heads, D] bf16 with contiguous heads; returns (T, heads, stride between tokens)."""
    if t.dtype != _BF16 or t.dim() != 3 or t.shape[2] != D or t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != D):
        raise TypeError(f"{name} must be a bf16 [T, heads, {D}] tensor with contiguous heads")
    return t.shape[0], t.shape[1], (t.stride(0) if t.shape[0] > 1 else t.shape[1] * D)


def cake_kv_append(cache, k, v, slots, positions=None, cos_sin=None, q=None, out_q=None, interleaved=False, ws=None, stream=None):
    """Writes k, v bf16 [T,Hkv,D] to `slots` (int64 [T], negative: skipped) of the cache; with cos_sin fp32 [positions, rot] (cosines,
    then sines) and positions int32 [T], keys and queries are rotated.  Returns the rotated queries (None without q); out_q may be q."""
    T, Hkv, k_stride = _heads(k, cache.D, "k")
    Tv, Hv, v_stride = _heads(v, cache.D, "v")
    if (Tv, Hv) != (T, Hkv) or Hkv != cache.Hkv:
        raise ValueError("k and v must be [T, Hkv, D] with the cache's Hkv")
    _dense(slots, torch.int64, (T,), "slots")
    rot, longest = 0, 0
    if cos_sin is not None:
        if positions is None or cos_sin.dim() != 2:
            raise ValueError("a rotation takes positions [T] and cos_sin [max_positions, rot]")
        longest, rot = cos_sin.shape
        _dense(cos_sin, torch.float32, (longest, rot), "cos_sin")
        _dense(positions, torch.int32, (T,), "positions")
    Hq, q_stride = 0, 0
    if q is not None:
        Tq, Hq, q_stride = _heads(q, cache.D, "q")
        if Tq != T:
            raise ValueError("q must have k's tokens")
        if out_q is None:
            out_q = torch.empty(T, Hq, cache.D, dtype=_BF16, device=q.device)
        _dense(out_q, _BF16, (T, Hq, cache.D), "out_q")
    else:
        out_q = None
    if ws is None:
        ws = alloc_append_workspace(cache.device)
    _buffer(ws, 0, "ws")
    _on(cache.device, k=k, v=v, q=q, out_q=out_q, slots=slots, positions=positions, cos_sin=cos_sin, ws=ws)
    fn = _load().cake_kv_append
    flags = CAKE_APPEND_INTERLEAVED if interleaved else 0
    _call(lambda *a: fn(*a, flags), "cake_kv_append", cache.device, stream, cache._ref, _p(k), k_stride, _p(v), v_stride, _p(q), q_stride, Hq,
          _p(out_q), _p(slots), _p(positions) if rot else None, _p(cos_sin) if rot else None, longest, rot, T, _p(ws), ws.numel())
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
    D, Hkv = cache.D, cache.Hkv
    if q.dtype != _BF16 or q.dim() != 3 or q.shape[2] != D or q.stride(2) != 1:
        raise TypeError(f"q must be a bf16 [B, Hq, {D}] tensor with contiguous rows")
    B, Hq, _ = q.shape
    if page_table.dtype != torch.int32 or page_table.dim() not in (2, 3) or (page_table.shape[-1] > 1 and page_table.stride(-1) != 1):
        raise TypeError("page_table must be int32 [B, max_pages] or [B, Hkv, max_pages] with contiguous rows")
    if seq_lens.dtype != torch.int32 or seq_lens.dim() not in (1, 2):
        raise TypeError("seq_lens must be int32 [B] or [B, Hkv]")
    if page_table.shape[0] != B or seq_lens.shape[0] != B or (page_table.dim() == 3 and page_table.shape[1] != Hkv) or \
            (seq_lens.dim() == 2 and seq_lens.shape[1] != Hkv):
        raise ValueError("page_table and seq_lens must have q's B (and the cache's Hkv where they are per head)")
    if out is None:
        out = torch.empty(B, Hq, D, dtype=_BF16, device=q.device)
    _dense(out, _BF16, (B, Hq, D), "out")
    if out_lse is None and want_lse:
        out_lse = torch.empty(B, Hq, dtype=torch.float32, device=q.device)
    if out_lse is not None:
        _dense(out_lse, torch.float32, (B, Hq), "out_lse")
    if ws is None:
        ws = alloc_decode_workspace(B, Hq, Hkv, D, q.device)
    _buffer(ws, 0, "ws")
    _on(cache.device, q=q, page_table=page_table, seq_lens=seq_lens, out=out, out_lse=out_lse, ws=ws)
    fn = _load().cake_paged_decode
    _call(fn, "cake_paged_decode", cache.device, stream, _p(q), q.stride(0), q.stride(1), cache._ref, _p(page_table), page_table.stride(0),
          page_table.stride(1) if page_table.dim() == 3 else 0, page_table.shape[-1], _p(seq_lens), seq_lens.stride(0),
          seq_lens.stride(1) if seq_lens.dim() == 2 else 0, B, Hq, 1.0 / math.sqrt(D) if scale is None else scale, window, _p(out),
          _p(out_lse), _p(ws), ws.numel())
    return out, out_lse
