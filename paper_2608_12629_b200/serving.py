"""ctypes binding of the serving operators (include/cake_serving.h): argument marshalling only.

Each function has the name of the C entry point it calls; PyTorch supplies device memory and the stream.  As in `binding`,
there is no fallback: a missing library, a wrong type or a refused shape raises.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import binding
from .binding import CakeError, _check

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


# The checks below are the calls' cost on the host, which small problems feel: plain attribute tests, no temporaries, one
# pass over the tensors.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(fn, where, index, *args):
    """fn(*args) with device `index` current; a refusal raises."""
    if index == _current_device():
        rc = fn(*args)
    else:
        with torch.cuda.device(index):
            rc = fn(*args)
    if rc != 0:
        raise CakeError(rc, where)


def _handle(stream, index):
    return _raw_stream(index) if stream is None else stream.cuda_stream


def _device(t):
    index = t.get_device()
    if index < 0:
        raise TypeError("the operators take CUDA tensors")
    return index


def _rows(t, dtype, name):
    """A matrix whose rows are contiguous; returns (rows, columns, stride between rows)."""
    if t.dtype is dtype and t.dim() == 2:
        n, c = t.shape
        s0, s1 = t.stride()
        if s1 == 1 or c <= 1:
            return n, c, (s0 if n > 1 else c)
    raise TypeError(f"{name} must be a {dtype} matrix with contiguous rows")


def _dense(t, dtype, shape, name, index):
    """Address of a contiguous tensor of this type and shape on device `index`."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{index}")
    return t.data_ptr()


def _same(t, name, index):
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{index}")
    return t.data_ptr()


def _scratch(ws, index):
    if ws.dtype is not torch.uint8 or not ws.is_contiguous():
        raise TypeError("ws must be a contiguous uint8 tensor")
    return _same(ws, "ws", index), ws.numel()


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
    index = _device(x)
    T, H, x_stride = _rows(x, _BF16, "x")
    shape = (T, H)
    r_stride, r_ptr, w_ptr, res_ptr, y_ptr, q_ptr, s_ptr = H, None, None, None, None, None, None
    if residual is not None:
        Tr, Hr, r_stride = _rows(residual, _BF16, "residual")
        if (Tr, Hr) != shape:
            raise ValueError("residual must have x's shape")
        r_ptr = _same(residual, "residual", index)
    if weight is not None:
        w_ptr = _dense(weight, _BF16, (H,), "weight", index)
    if out_residual is None and (residual is not None if want_residual is None else want_residual):
        out_residual = torch.empty(T, H, dtype=_BF16, device=x.device)
    if out_residual is not None:
        res_ptr = _dense(out_residual, _BF16, shape, "out_residual", index)
    if out_y is None and want_y:
        out_y = torch.empty(T, H, dtype=_BF16, device=x.device)
    if out_y is not None:
        y_ptr = _dense(out_y, _BF16, shape, "out_y", index)
    if out_q is None and want_q:
        out_q = torch.empty(T, H, dtype=_E4M3, device=x.device)
    if out_q is not None:
        n = 1 if group == 0 else -(-H // 128)
        if out_scale is None:
            out_scale = torch.empty(T, n, dtype=torch.float32, device=x.device)
        q_ptr = _dense(out_q, _E4M3, shape, "out_q", index)
        s_ptr = _dense(out_scale, torch.float32, (T, n), "out_scale", index)
    _call(_load().cake_rmsnorm_quant, "cake_rmsnorm_quant", index, x.data_ptr(), x_stride, r_ptr, r_stride, w_ptr, T, H, eps,
          group, res_ptr, y_ptr, q_ptr, s_ptr, _handle(stream, index), flags)
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
    index = _device(X)
    M, K, x_stride = _rows(X, _E4M3, "X")
    N, Kw, w_stride = _rows(W, _E4M3, "W")
    if K != Kw:
        raise ValueError("X must be [M,K] and W [N,K]")
    nk = -(-K // 128)
    xs_ptr = _dense(x_scale, torch.float32, (M, nk), "x_scale", index)
    ws_ptr = _dense(w_scale, torch.float32, (-(-N // 128), nk), "w_scale", index)
    if out is None:
        if out_dtype not in (_BF16, torch.float32):
            raise TypeError("out_dtype must be torch.bfloat16 or torch.float32")
        out = torch.empty(M, N, dtype=out_dtype, device=X.device)
    fp32 = out.dtype is torch.float32
    Mo, No, out_stride = _rows(out, torch.float32 if fp32 else _BF16, "out")
    if Mo != M or No != N:
        raise TypeError("out must be a bf16 or fp32 [M,N] matrix")
    if ws is None:
        ws = alloc_gemm_workspace(M, N, K, X.device)
    buf, size = _scratch(ws, index)
    _call(_load().cake_gemm_fp8, "cake_gemm_fp8", index, X.data_ptr(), x_stride, xs_ptr, _same(W, "W", index), w_stride, ws_ptr, M, N, K,
          _same(out, "out", index), out_stride, buf, size, _handle(stream, index), CAKE_GEMM_OUT_FP32 if fp32 else 0)
    return out


# --------------------------------------------------------------------------------------------------------------- cache
class PagedCache:
    """A paged cache of keys and values: k and v [num_pages, page_size, Hkv, D], bf16 or e4m3, D contiguous, any other strides (a
    cache held head by head inside a page is passed as a transposed view).  k_scale, v_scale: fp32 [Hkv] or None (ones): an
    element x is held as x / scale.  Keeps the tensors alive; holds no copy."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        self.index = _device(k)
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in (_BF16, _E4M3):
            raise TypeError("k and v must be bf16 or e4m3 [num_pages, page_size, Hkv, D] of the same shape")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise TypeError("the last dimension of k and v must be contiguous")
        pages, page, Hkv, D = k.shape
        ptrs = [None if t is None else _dense(t, torch.float32, (Hkv,), name, self.index) for name, t in (("k_scale", k_scale), ("v_scale", v_scale))]
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.page_size, self.Hkv, self.D = pages, page, Hkv, D
        self._struct = _CacheStruct(k.data_ptr(), _same(v, "v", self.index), *ptrs, pages, k.stride(0), k.stride(1), k.stride(2), v.stride(0),
                                    v.stride(1), v.stride(2), page, Hkv, D, CAKE_KV_E4M3 if k.dtype == _E4M3 else CAKE_KV_BF16)
        self._ref = ctypes.byref(self._struct)

    @property
    def device(self):
        return self.k.device


def alloc_append_workspace(device) -> torch.Tensor:
    """A workspace for cake_kv_append (its device status), zeroed."""
    return _workspace(CAKE_SERVING_HEADER_BYTES, device)


def _heads(t, D, name, index):
    """[T, heads, D] bf16 with contiguous heads; returns (T, heads, stride between tokens, address)."""
    if t.dtype is _BF16 and t.dim() == 3:
        T, H, d = t.shape
        s0, s1, s2 = t.stride()
        if d == D and s2 == 1 and (s1 == D or H <= 1):
            return T, H, (s0 if T > 1 else H * D), _same(t, name, index)
    raise TypeError(f"{name} must be a bf16 [T, heads, {D}] tensor with contiguous heads")


def cake_kv_append(cache, k, v, slots, positions=None, cos_sin=None, q=None, out_q=None, interleaved=False, ws=None, stream=None):
    """Writes k, v bf16 [T,Hkv,D] to `slots` (int64 [T], negative: skipped) of the cache; with cos_sin fp32 [positions, rot] (cosines,
    then sines) and positions int32 [T], keys and queries are rotated.  Returns the rotated queries (None without q); out_q may be q."""
    D, index = cache.D, cache.index
    T, Hkv, k_stride, k_ptr = _heads(k, D, "k", index)
    Tv, Hv, v_stride, v_ptr = _heads(v, D, "v", index)
    if Tv != T or Hv != Hkv or Hkv != cache.Hkv:
        raise ValueError("k and v must be [T, Hkv, D] with the cache's Hkv")
    slot_ptr = _dense(slots, torch.int64, (T,), "slots", index)
    rot, longest, pos_ptr, table_ptr = 0, 0, None, None
    if cos_sin is not None:
        if positions is None or cos_sin.dim() != 2:
            raise ValueError("a rotation takes positions [T] and cos_sin [max_positions, rot]")
        longest, rot = cos_sin.shape
        table_ptr = _dense(cos_sin, torch.float32, (longest, rot), "cos_sin", index)
        pos_ptr = _dense(positions, torch.int32, (T,), "positions", index)
    Hq, q_stride, q_ptr, out_ptr = 0, 0, None, None
    if q is not None:
        Tq, Hq, q_stride, q_ptr = _heads(q, D, "q", index)
        if Tq != T:
            raise ValueError("q must have k's tokens")
        if out_q is None:
            out_q = torch.empty(T, Hq, D, dtype=_BF16, device=q.device)
        out_ptr = _dense(out_q, _BF16, (T, Hq, D), "out_q", index)
    else:
        out_q = None
    if ws is None:
        ws = alloc_append_workspace(k.device)
    buf, size = _scratch(ws, index)
    _call(_load().cake_kv_append, "cake_kv_append", index, cache._ref, k_ptr, k_stride, v_ptr, v_stride, q_ptr, q_stride, Hq, out_ptr, slot_ptr,
          pos_ptr, table_ptr, longest, rot, T, buf, size, _handle(stream, index), CAKE_APPEND_INTERLEAVED if interleaved else 0)
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
    D, Hkv, index = cache.D, cache.Hkv, cache.index
    if q.dtype is not _BF16 or q.dim() != 3:
        raise TypeError("q must be a bf16 [B, Hq, D] tensor")
    B, Hq, Dq = q.shape
    q0, q1, q2 = q.stride()
    if Dq != D or q2 != 1:
        raise TypeError(f"q must be a bf16 [B, Hq, {D}] tensor with contiguous rows")
    if page_table.dtype is not torch.int32 or seq_lens.dtype is not torch.int32:
        raise TypeError("page_table and seq_lens must be int32")
    table_shape, table_strides = page_table.shape, page_table.stride()
    lens_shape, lens_strides = seq_lens.shape, seq_lens.stride()
    tables, lengths = len(table_shape), len(lens_shape)
    if tables not in (2, 3) or lengths not in (1, 2) or (table_shape[-1] > 1 and table_strides[-1] != 1):
        raise TypeError("page_table must be [B, max_pages] or [B, Hkv, max_pages] with contiguous rows, seq_lens [B] or [B, Hkv]")
    if table_shape[0] != B or lens_shape[0] != B or (tables == 3 and table_shape[1] != Hkv) or (lengths == 2 and lens_shape[1] != Hkv):
        raise ValueError("page_table and seq_lens must have q's B (and the cache's Hkv where they are per head)")
    if out is None:
        out = torch.empty(B, Hq, D, dtype=_BF16, device=q.device)
    out_ptr = _dense(out, _BF16, (B, Hq, D), "out", index)
    if out_lse is None and want_lse:
        out_lse = torch.empty(B, Hq, dtype=torch.float32, device=q.device)
    lse_ptr = None if out_lse is None else _dense(out_lse, torch.float32, (B, Hq), "out_lse", index)
    if ws is None:
        ws = alloc_decode_workspace(B, Hq, Hkv, D, q.device)
    buf, size = _scratch(ws, index)
    _call(_load().cake_paged_decode, "cake_paged_decode", index, _same(q, "q", index), q0, q1, cache._ref, _same(page_table, "page_table", index),
          table_strides[0], table_strides[1] if tables == 3 else 0, table_shape[-1], _same(seq_lens, "seq_lens", index), lens_strides[0],
          lens_strides[1] if lengths == 2 else 0, B, Hq, 1.0 / math.sqrt(D) if scale is None else scale, window, out_ptr, lse_ptr, buf, size,
          _handle(stream, index))
    return out, out_lse
