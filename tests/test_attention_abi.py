"""Attention of many tokens, norm with append, reading back: what the host can refuse needs no device."""
import ctypes

import pytest

import paper_2608_12629_b200 as cake
from paper_2608_12629_b200 import build as cake_build
from paper_2608_12629_b200 import serving


@pytest.fixture(scope="module")
def L():
    cake_build.build_library()
    return serving._load()


def cache(**more):
    c = serving._CacheStruct(4096, 4096, None, None, 4, 16 * 128, 128, 128, 16 * 128, 128, 128, 16, 1, 128, cake.CAKE_KV_BF16)
    for k, v in more.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def test_workspace_sizes():
    assert cake.cake_attention_workspace_bytes(8, 2, 64) < cake.cake_attention_workspace_bytes(8, 2, 128)
    for bad, code in (((3, 2, 64), cake.CAKE_ERR_SHAPE), ((0, 1, 64), cake.CAKE_ERR_SHAPE), ((1, 0, 64), cake.CAKE_ERR_SHAPE), ((1, 1, 80), cake.CAKE_ERR_UNSUPPORTED)):
        with pytest.raises(cake.CakeError) as e:
            cake.cake_attention_workspace_bytes(*bad)
        assert e.value.code == code


def test_prompt_refusals(L):
    def call(q=4096, qs=512, qh=128, k=4096, ks=256, kh=128, v=4096, vs=256, vh=128, st=4096, kst=None, B=2, T=9, Tk=9, Hq=4, Hkv=2, D=128, window=0, out=4096,
             lse=None, buf=4096, n=1 << 30, flags=1):
        return L.cake_prompt_attention(q, qs, qh, k, ks, kh, v, vs, vh, st, kst, B, T, Tk, Hq, Hkv, D, 0.1, window, out, lse, buf, n, None, flags)
    for name in ("q", "k", "v", "st", "out", "buf"):
        assert call(**{name: None}) == cake.CAKE_ERR_NULL, name
    assert call(B=-1) == call(T=-1) == call(Tk=-1) == call(T=2 ** 31 - 1) == call(Hq=3) == call(Hq=0) == call(Hkv=0) == call(window=-1) == cake.CAKE_ERR_SHAPE
    assert call(qs=0) == call(qh=64) == call(ks=120) == call(vh=0) == call(ks=-256) == cake.CAKE_ERR_SHAPE
    assert call(q=4104) == call(k=4100) == call(v=4098) == call(qs=516) == call(kh=132) == call(vs=260) == cake.CAKE_ERR_ALIGN
    assert call(out=4097) == call(lse=4098) == call(st=4098) == call(kst=4098) == call(buf=4100) == cake.CAKE_ERR_ALIGN
    assert call(D=80) == call(flags=2) == call(flags=0, window=4) == cake.CAKE_ERR_UNSUPPORTED
    assert call(n=cake.cake_attention_workspace_bytes(4, 2, 128) - 1) == cake.CAKE_ERR_WORKSPACE
    assert call(B=0, q=None) == call(T=0, q=None) == cake.CAKE_OK


def test_chunk_refusals(L):
    def call(c=None, q=4096, qs=512, qh=128, table=4096, ts=4, width=4, lens=4096, st=4096, B=2, T=9, Hq=4, window=0, out=4096, lse=None, buf=4096, n=1 << 30):
        return L.cake_paged_chunk(q, qs, qh, c or cache(), table, ts, 0, width, lens, 1, 0, st, B, T, Hq, 0.1, window, out, lse, buf, n, None)
    for name in ("q", "table", "lens", "st", "out", "buf"):
        assert call(**{name: None}) == cake.CAKE_ERR_NULL, name
    assert call(B=-1) == call(T=-1) == call(Hq=0) == call(window=-1) == call(width=-1) == call(width=2 ** 30) == call(ts=-1) == call(qs=64) == cake.CAKE_ERR_SHAPE
    assert call(c=cache(Hkv=2), Hq=3) == cake.CAKE_ERR_SHAPE
    assert call(q=4104) == call(qh=130) == call(out=4097) == call(lse=4098) == call(buf=4100) == call(table=4097) == call(lens=4097) == call(st=4097) == cake.CAKE_ERR_ALIGN
    assert call(c=cache(D=72)) == call(c=cache(type=3)) == cake.CAKE_ERR_UNSUPPORTED
    assert call(n=cake.CAKE_SERVING_HEADER_BYTES) == cake.CAKE_ERR_WORKSPACE
    assert call(B=0, q=None) == call(T=0, q=None) == cake.CAKE_OK


def test_qk_norm_refusals(L):
    def call(c=None, q=4096, qs=256, Hq=2, k=4096, ks=128, v=4096, vs=128, wq=None, wk=None, oq=4096, ok=None, slots=4096, pos=4096, cs=4096, longest=8, rot=128, T=3,
             buf=4096, n=1 << 20, flags=0):
        return L.cake_qk_norm_append(c or cache(), q, qs, Hq, k, ks, v, vs, wq, wk, 1e-6, oq, ok, slots, pos, cs, longest, rot, T, buf, n, None, flags)
    for name in ("q", "k", "v", "oq", "slots", "pos", "cs", "buf"):
        assert call(**{name: None}) == cake.CAKE_ERR_NULL, name
    assert call(rot=127) == call(rot=130) == call(rot=-2) == call(ks=127) == call(vs=1) == call(qs=255) == call(T=-1) == call(longest=0) == call(Hq=0) == cake.CAKE_ERR_SHAPE
    assert call(q=4097) == call(wq=4097) == call(wk=4099) == call(ok=4097) == call(oq=4097) == call(slots=4100) == call(buf=4100) == cake.CAKE_ERR_ALIGN
    assert call(n=256) == cake.CAKE_ERR_WORKSPACE and call(flags=2) == cake.CAKE_ERR_UNSUPPORTED and call(c=cache(D=80)) == cake.CAKE_ERR_UNSUPPORTED
    assert call(T=0, q=None) == cake.CAKE_OK


def test_read_refusals(L):
    def call(c=None, slots=4096, N=3, k=4096, v=4096, s=128, hs=128, buf=4096, n=1 << 20):
        return L.cake_kv_read(c or cache(), slots, N, k, v, s, hs, buf, n, None)
    assert call(slots=None) == call(buf=None) == call(c=cache(k=None)) == cake.CAKE_ERR_NULL
    assert call(N=-1) == call(s=64) == call(c=cache(Hkv=2), hs=64) == cake.CAKE_ERR_SHAPE
    assert call(slots=4100) == call(k=4104) == call(v=4098) == call(s=132) == call(c=cache(Hkv=2), hs=132) == call(buf=4100) == cake.CAKE_ERR_ALIGN
    assert call(n=256) == cake.CAKE_ERR_WORKSPACE and call(c=cache(D=80)) == cake.CAKE_ERR_UNSUPPORTED
    assert call(N=0, slots=None) == call(k=None, v=None) == cake.CAKE_OK
