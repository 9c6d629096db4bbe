"""The serving operators' part of the C ABI: exported, declared and bound alike; what the host can refuse needs no device."""
import ctypes
import os
import re

import pytest

import paper_2608_12629_b200 as cake
from paper_2608_12629_b200 import build as cake_build
from paper_2608_12629_b200 import serving

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def L():
    cake_build.build_library()
    return serving._load()


def header():
    return open(os.path.join(ROOT, "include", "cake_serving.h")).read()


def test_header_library_and_binding_agree(L):
    names = sorted(set(re.findall(r"CAKE_API\s+[\w\s\*]+?\b(cake_\w+)\s*\(", header())))
    assert names == sorted(cake.SERVING_EXPORTS)
    for n in names:
        assert hasattr(L, n)
    assert int(re.search(r"CAKE_SERVING_HEADER_BYTES (\d+)", header()).group(1)) == cake.CAKE_SERVING_HEADER_BYTES


def test_marshalling_module_refuses_what_is_no_cuda_tensor(L):
    import torch
    cake_build.build_extension()
    x = torch.zeros(2, 8, dtype=torch.bfloat16)
    for bad in (x, x.float(), None, 3, x.view(-1)):
        with pytest.raises((TypeError, AttributeError, IndexError)):
            cake.cake_rmsnorm_quant(bad)
    with pytest.raises(TypeError):
        serving._native().gemm_fp8(x, x)                 # a wrong number of arguments
    with pytest.raises(TypeError):
        serving._native().rmsnorm_quant(*[x] * 11)
    with pytest.raises(TypeError):
        cake.PagedCache(x, x)
    with pytest.raises(TypeError):
        cake.PagedCache(*[torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16)] * 2)


def test_workspace_sizes_need_no_device():
    assert cake.cake_gemm_fp8_workspace_bytes(1, 128, 128) >= cake.CAKE_SERVING_HEADER_BYTES
    assert cake.cake_gemm_fp8_workspace_bytes(0, 1, 16) >= cake.CAKE_SERVING_HEADER_BYTES
    assert cake.cake_gemm_fp8_workspace_bytes(256, 256, 8192) > cake.cake_gemm_fp8_workspace_bytes(8192, 8192, 8192)
    assert cake.cake_paged_decode_workspace_bytes(1, 1, 1, 64) < cake.cake_paged_decode_workspace_bytes(1, 16, 1, 256)
    for bad in [(-1, 8, 16), (1, 0, 16), (1, 8, 0), (2 ** 31, 8, 16)]:
        with pytest.raises(cake.CakeError) as e:
            cake.cake_gemm_fp8_workspace_bytes(*bad)
        assert e.value.code == cake.CAKE_ERR_SHAPE
    for bad, code in [((1, 3, 2, 64), cake.CAKE_ERR_SHAPE), ((1, 0, 1, 64), cake.CAKE_ERR_SHAPE), ((-1, 1, 1, 64), cake.CAKE_ERR_SHAPE),
                      ((1, 1, 1, 80), cake.CAKE_ERR_UNSUPPORTED)]:
        with pytest.raises(cake.CakeError) as e:
            cake.cake_paged_decode_workspace_bytes(*bad)
        assert e.value.code == code


def test_no_product_needs_more_than_the_most(L):
    """A buffer for any number of rows: the size needed is no growing function of them."""
    most = cake.CAKE_GEMM_FP8_MOST_WORKSPACE_BYTES
    assert int(re.search(r"CAKE_GEMM_FP8_MOST_WORKSPACE_BYTES (\d+)", header()).group(1)) == most
    assert cake.cake_gemm_fp8_workspace_bytes(256, 4096, 4096) > cake.cake_gemm_fp8_workspace_bytes(8192, 4096, 4096)
    ms = [1, 16, 64, 65, 128, 200, 256, 257, 384, 512, 517, 768, 1000, 1024, 2048, 4096, 5000, 18944, 100000]
    ns = [1, 127, 128, 129, 256, 300, 512, 640, 1000, 1024, 1280, 2048, 2624, 4096, 6144, 8192, 9472, 18944, 18945, 100000]
    sizes = [cake.cake_gemm_fp8_workspace_bytes(m, n, k) for m in ms for n in ns for k in (16, 128, 512, 1024, 4096, 8192, 14336, 131072)]
    assert max(sizes) <= most and max(sizes) > 0.9 * most


def cache(**more):
    c = serving._CacheStruct(4096, 4096, None, None, 4, 16 * 128, 128, 128, 16 * 128, 128, 128, 16, 1, 128, cake.CAKE_KV_BF16)
    for k, v in more.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def test_norm_refusals(L):
    def call(x=4096, xs=64, r=None, rs=0, T=2, H=64, group=128, y=None, q=4096, sc=4096, flags=0, w=None):
        return L.cake_rmsnorm_quant(x, xs, r, rs, w, T, H, 1e-6, group, None, y, q, sc, None, flags)
    assert call(x=None) == cake.CAKE_ERR_NULL and call(q=None, sc=None) == cake.CAKE_ERR_NULL and call(sc=None) == cake.CAKE_ERR_NULL
    assert call(T=-1) == cake.CAKE_ERR_SHAPE and call(H=0) == cake.CAKE_ERR_SHAPE and call(xs=63) == cake.CAKE_ERR_SHAPE
    assert call(r=4096, rs=3) == cake.CAKE_ERR_SHAPE
    assert call(group=32) == cake.CAKE_ERR_UNSUPPORTED and call(flags=2) == cake.CAKE_ERR_UNSUPPORTED
    assert call(H=32769, xs=32769) == cake.CAKE_ERR_UNSUPPORTED
    assert call(x=4097) == cake.CAKE_ERR_ALIGN and call(w=4097) == cake.CAKE_ERR_ALIGN and call(sc=4098) == cake.CAKE_ERR_ALIGN
    assert call(T=0, x=None) == cake.CAKE_OK


def test_gemm_refusals(L):
    def call(x=4096, ldx=128, xs=4096, w=4096, ldw=128, ws=4096, M=4, N=8, K=128, out=4096, ldo=8, buf=4096, n=1 << 30, flags=0):
        return L.cake_gemm_fp8(x, ldx, xs, w, ldw, ws, M, N, K, out, ldo, buf, n, None, flags)
    for name in ("x", "xs", "w", "ws", "out", "buf"):
        assert call(**{name: None}) == cake.CAKE_ERR_NULL, name
    assert call(M=-1) == call(N=0) == call(K=0, ldx=0) == call(ldx=112) == call(ldw=112) == call(ldo=7) == cake.CAKE_ERR_SHAPE
    assert call(x=4100) == call(w=4104) == call(ldx=136) == call(ldw=136) == call(K=120) == call(out=4097) == call(buf=4100) == cake.CAKE_ERR_ALIGN
    assert call(n=cake.CAKE_SERVING_HEADER_BYTES - 1) == cake.CAKE_ERR_WORKSPACE
    assert call(flags=4) == cake.CAKE_ERR_UNSUPPORTED
    assert call(M=0, x=None) == cake.CAKE_OK


def test_append_refusals(L):
    def call(c=None, k=4096, ks=128, v=4096, vs=128, q=None, qs=0, Hq=0, oq=None, slots=4096, pos=4096, cs=4096, longest=8, rot=128, T=3,
             buf=4096, n=1 << 20, flags=0):
        return L.cake_kv_append(c or cache(), k, ks, v, vs, q, qs, Hq, oq, slots, pos, cs, longest, rot, T, buf, n, None, flags)
    for name in ("k", "v", "slots", "pos", "cs", "buf"):
        assert call(**{name: None}) == cake.CAKE_ERR_NULL, name
    assert call(q=4096, qs=128, Hq=1) == cake.CAKE_ERR_NULL
    assert call(rot=127) == call(rot=130) == call(rot=-2) == call(ks=127) == call(vs=1) == call(T=-1) == call(longest=0) == cake.CAKE_ERR_SHAPE
    assert call(q=4096, qs=127, Hq=1, oq=4096) == cake.CAKE_ERR_SHAPE
    assert call(n=256) == cake.CAKE_ERR_WORKSPACE and call(buf=4100) == cake.CAKE_ERR_ALIGN and call(slots=4100) == cake.CAKE_ERR_ALIGN
    assert call(flags=2) == cake.CAKE_ERR_UNSUPPORTED
    assert call(c=cache(k=None)) == cake.CAKE_ERR_NULL
    assert call(c=cache(D=80)) == call(c=cache(type=2)) == cake.CAKE_ERR_UNSUPPORTED
    assert call(c=cache(page_size=0)) == call(c=cache(num_pages=0)) == call(c=cache(Hkv=0)) == call(c=cache(k_page_stride=-8)) == cake.CAKE_ERR_SHAPE
    assert call(c=cache(k=4104)) == call(c=cache(v_token_stride=132)) == call(c=cache(type=1, k_head_stride=136)) == cake.CAKE_ERR_ALIGN
    assert call(T=0, k=None) == cake.CAKE_OK


def test_decode_refusals(L):
    def call(c=None, q=4096, table=4096, width=4, lens=4096, B=2, Hq=2, window=0, out=4096, lse=None, buf=4096, n=1 << 30, ts=4, qs=256):
        return L.cake_paged_decode(q, qs, 128, c or cache(), table, ts, 0, width, lens, 1, 0, B, Hq, 0.1, window, out, lse, buf, n, None)
    for name in ("q", "table", "lens", "out", "buf"):
        assert call(**{name: None}) == cake.CAKE_ERR_NULL, name
    assert call(B=-1) == call(Hq=0) == call(window=-1) == call(width=-1) == call(width=2 ** 30) == call(ts=-1) == call(qs=-1) == cake.CAKE_ERR_SHAPE
    assert call(c=cache(Hkv=2), Hq=3) == cake.CAKE_ERR_SHAPE
    assert call(n=cake.CAKE_SERVING_HEADER_BYTES) == cake.CAKE_ERR_WORKSPACE
    assert call(q=4097) == call(out=4097) == call(lse=4098) == call(buf=4100) == call(table=4097) == cake.CAKE_ERR_ALIGN
    assert call(c=cache(D=72)) == cake.CAKE_ERR_UNSUPPORTED
    assert call(B=0, q=None) == cake.CAKE_OK
