"""Norm, rotation and append in one pass, and reading a cache back, against plain implementations in 64 bits.

Tolerances, from the arithmetic alone: sum of D <= 256 squares in 32 bits, the reciprocal root (2 ulp), three products and the rotation's
three roundings: (D / 16 + 16) 2^-23 < 2^-18 of |a| + |b| (the pair that rotates), then half a step of the output: bf16 2^-8, e4m3 2^-4
and 2^-10 of the scale.  Reading back is exact but for one rounding of a product to bf16.
"""
import pytest
import torch

import paper_2608_12629_b200 as cake

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
REL = 2.0 ** -18


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=BF16):
    return torch.empty(*shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def made(x, w, pos, table, pairs, eps):
    """x [T, H, D] -> normed and rotated, and |a| + |b| of every element's pair, in 64 bits."""
    x = x.double()
    y = x / (x.square().mean(2, keepdim=True) + eps).sqrt()
    if w is not None:
        y = y * w.double()
    size = y.abs()
    if table is not None:
        rot = table.shape[1]
        c, s = (t[:, None].double() for t in table[pos.long()].chunk(2, 1))
        ia, ib = (torch.arange(0, rot, 2), torch.arange(1, rot, 2)) if pairs else (torch.arange(rot // 2), torch.arange(rot // 2, rot))
        a, b = y[..., ia], y[..., ib]
        y, size = y.clone(), size.clone()
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return y, size


def close(got, want, bound, what):
    err = (got.double() - want).abs()
    assert not (~(err <= bound)).any(), f"{what}: worst {float((err / bound).max()):.3g} bounds"


def cache_of(seed, pages, page, Hkv, D, kv, by_head=False, filled=False):
    shape = (pages, Hkv, page, D) if by_head else (pages, page, Hkv, D)
    dtype = E4M3 if kv == "e4m3" else BF16
    g = gen(seed)
    k, v = ((normal(g, *shape, std=60.0 if kv == "e4m3" else 1.0, dtype=dtype) if filled else torch.zeros(*shape, dtype=dtype, device=DEV)) for _ in range(2))
    if by_head:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    scales = [torch.empty(Hkv, device=DEV).uniform_(0.01, 0.03, generator=g) if kv == "e4m3" else None for _ in range(2)]
    return cake.PagedCache(k, v, *scales)


def rotary(rot, longest=500):
    if not rot:
        return None
    angle = torch.arange(longest, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def check_cache(cache, slots, want_k, size_k, v):
    """Slots written hold the keys and values; all others are as they were (zero)."""
    kept = slots >= 0
    page, off = slots[kept] // cache.page_size, slots[kept] % cache.page_size
    for got, want, size, scale in ((cache.k, want_k, size_k, cache.k_scale), (cache.v, v.double(), v.double().abs(), cache.v_scale)):
        got = got.float()
        rows = got[page, off].double()
        if scale is None:
            close(rows, want[kept], 2.0 ** -8 * 1.01 * want[kept].abs() + REL * size[kept] + 1e-38, "cache")
        else:
            sc = scale.double()[None, :, None]
            clipped = (want[kept] / sc).clamp(-448, 448)
            close(rows, clipped, 2.0 ** -4 * 1.01 * clipped.abs() + 2 * REL * size[kept] / sc + 2.0 ** -10 * 1.01, "cache")
        rest = torch.ones(got.shape[:2], dtype=torch.bool, device=DEV)
        rest[page, off] = False
        assert (got[rest] == 0).all()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,rot,pairs", [(64, 64, False), (64, 16, True), (96, 96, False), (96, 32, False), (128, 128, False), (128, 128, True), (128, 64, False),
                                         (128, 0, False), (256, 256, True), (256, 64, False), (128, 40, True), (128, 24, False), (64, 6, True), (96, 10, False)])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 1, 1), (5, 6, 2), (200, 32, 8)])
def test_qk_norm(kv, D, rot, pairs, T, Hq, Hkv):
    g = gen(D + rot + T)
    rows = normal(g, T, Hq + 2 * Hkv, D, std=2.0)
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    wq, wk = normal(g, D, std=0.3) + 1, normal(g, D, std=0.3) + 1
    cache = cache_of(1, 40, 16, Hkv, D, kv, by_head=T == 5)
    slots = torch.randperm(640, device=DEV, generator=g)[:T].clone()
    slots[2::5] = -1
    table = rotary(rot)
    pos = torch.randint(0, 500, (T,), device=DEV, generator=g, dtype=torch.int32)
    ws = cake.alloc_append_workspace(DEV)
    got_q, got_k = cake.cake_qk_norm_append(cache, q, k, v, slots, wq, wk, pos if rot else None, table, interleaved=pairs, want_k=True, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK
    want_q, size_q = made(q, wq, pos, table, pairs, 1e-6)
    want_k, size_k = made(k, wk, pos, table, pairs, 1e-6)
    close(got_q, want_q, 2.0 ** -8 * 1.01 * want_q.abs() + REL * size_q + 1e-38, "q")
    close(got_k, want_k, 2.0 ** -8 * 1.01 * want_k.abs() + REL * size_k + 1e-38, "k")
    check_cache(cache, slots, want_k, size_k, v)


@pytest.mark.parametrize("offset,stride", [(0, 8), (1, 8), (0, 3)])
def test_qk_norm_alignments_and_in_place(offset, stride):
    """Sources that are not 16-byte aligned take another path; the results differ by roundings at most."""
    g = gen(3)
    T, Hq, Hkv, D = 300, 4, 2, 128
    width = (Hq + 2 * Hkv) * D
    buf = normal(g, T, width + stride)[:, offset:offset + width] if stride != 8 or offset else normal(g, T, width)
    rows = [buf[:, i * D:j * D].unflatten(1, (j - i, D)) for i, j in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv))]
    table, pos = rotary(D), torch.arange(T, device=DEV, dtype=torch.int32)
    cache = cache_of(1, 40, 16, Hkv, D, "bf16")
    slots = torch.arange(T, device=DEV)
    q, none = cake.cake_qk_norm_append(cache, *rows, slots, positions=pos, cos_sin=table, eps=1e-3)
    assert none is None
    want_q, size_q = made(rows[0], None, pos, table, False, 1e-3)
    want_k, size_k = made(rows[1], None, pos, table, False, 1e-3)
    close(q, want_q, 2.0 ** -8 * 1.01 * want_q.abs() + REL * size_q + 1e-38, "q")
    check_cache(cache, slots, want_k, size_k, rows[2])
    q2, k2 = rows[0].contiguous(), rows[1].contiguous()
    cake.cake_qk_norm_append(cache, q2, k2, rows[2], slots, positions=pos, cos_sin=table, eps=1e-3, out_q=q2, out_k=k2)
    close(q2, want_q, 2.0 ** -8 * 1.01 * want_q.abs() + REL * size_q + 1e-38, "q in place")
    close(k2, want_k, 2.0 ** -8 * 1.01 * want_k.abs() + REL * size_k + 1e-38, "k in place")


def test_qk_norm_rows_of_zeros_and_values_that_are_not_finite():
    g = gen(4)
    q, k, v = normal(g, 6, 2, 64), normal(g, 6, 1, 64), normal(g, 6, 1, 64)
    q[0], k[1] = 0, 0
    q[2, 0, 3], k[3, 0, 5] = float("nan"), float("inf")
    cache = cache_of(1, 2, 16, 1, 64, "bf16")
    oq, ok = cake.cake_qk_norm_append(cache, q, k, v, torch.arange(6, device=DEV), want_k=True)
    assert (oq[0] == 0).all() and (ok[1] == 0).all() and torch.isnan(oq[2, 0]).all() and torch.isfinite(oq[2, 1]).all()
    assert torch.isnan(ok[3, 0, 5]) and (ok[3, 0, :5] == 0).all() and torch.isfinite(ok[4:]).all()


def test_qk_norm_indices_out_of_range():
    g = gen(5)
    T, D = 40, 64
    q, k, v = normal(g, T, 2, D), normal(g, T, 1, D), normal(g, T, 1, D)
    for aligned in (True, False):
        cache = cache_of(1, 4, 16, 1, D, "bf16")
        slots = torch.arange(T, device=DEV)
        slots[7] = 64                               # one behind the cache
        pos = torch.zeros(T, dtype=torch.int32, device=DEV)
        pos[9], pos[11] = 500, -1
        oq, ok = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
        ws = cake.alloc_append_workspace(DEV)
        src = [x if aligned else torch.cat([x.view(T, -1), x.view(T, -1)[:, :1]], 1)[:, :-1].unflatten(1, x.shape[1:]) for x in (q, k, v)]
        cake.cake_qk_norm_append(cache, *src, slots, positions=pos, cos_sin=rotary(D), out_q=oq, out_k=ok, ws=ws)
        assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
        assert (oq[9] == 9).all() and (ok[11] == 9).all() and (ok[7] != 9).any()
        flat = cache.k.reshape(64, D)
        assert (flat[[7, 9, 11]] == 0).all() and (flat[8] != 0).any() and (flat[40:] == 0).all()


def test_qk_norm_no_tokens_and_refusals():
    q, k = torch.zeros(3, 2, 64, dtype=BF16, device=DEV), torch.zeros(3, 1, 64, dtype=BF16, device=DEV)
    cache = cache_of(1, 2, 16, 1, 64, "bf16")
    slots = torch.arange(3, device=DEV)
    assert cake.cake_qk_norm_append(cache, q[:0], k[:0], k[:0], slots[:0])[0].shape == (0, 2, 64)
    with pytest.raises(ValueError):
        cake.cake_qk_norm_append(cache, q[:2], k, k, slots)
    with pytest.raises(ValueError):
        cake.cake_qk_norm_append(cache, q, q, q, slots)
    with pytest.raises(ValueError):
        cake.cake_qk_norm_append(cache, q, k, k, slots, cos_sin=rotary(64))
    for bad in (dict(slots=slots.int()), dict(q_weight=torch.ones(64, device=DEV)), dict(k_weight=torch.ones(2, 64, dtype=BF16, device=DEV)), dict(q=q.float()),
                dict(out_k=torch.zeros(3, 2, 64, dtype=BF16, device=DEV))):
        with pytest.raises(TypeError):
            cake.cake_qk_norm_append(**{**dict(cache=cache, q=q, k=k, v=k, slots=slots), **bad})


# -------------------------------------------------------------------------------------------------------------- read
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hkv", [(64, 1), (96, 3), (128, 8), (256, 2)])
@pytest.mark.parametrize("N,page", [(1, 16), (37, 1), (1000, 100)])
def test_read(kv, D, Hkv, N, page):
    cache = cache_of(D + N, 1200 // page, page, Hkv, D, kv, by_head=N == 37, filled=True)
    g = gen(N)
    slots = torch.randint(-1, cache.num_pages * page, (N,), device=DEV, generator=g)
    kept = slots >= 0
    ws = cake.alloc_append_workspace(DEV)
    k, v = cake.cake_kv_read(cache, slots, ws=ws)
    for got, held, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        want = held.float()[slots.clamp(min=0) // page, slots.clamp(min=0) % page]
        want = want * (scale[None, :, None] if scale is not None else 1.0) * kept[:, None, None]
        assert got.shape == (N, Hkv, D) and torch.equal(got, want.to(BF16))      # (one product in 32 bits, one rounding)
    kh, none = cake.cake_kv_read(cache, slots, by_head=True, want_v=False)
    assert none is None and torch.equal(kh, k.transpose(0, 1))
    none, vh = cake.cake_kv_read(cache, slots, by_head=True, want_k=False)
    assert none is None and torch.equal(vh, v.transpose(0, 1))
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("N", [1, 50, 3000])
def test_read_to_every_allowed_alignment(kv, N):
    """Outputs are 16-byte aligned: 16 bytes behind a multiple of 32 they hold the same, and nothing beside them is touched."""
    cache = cache_of(5, 40, 100, 3, 96, kv, filled=True)
    slots = torch.randint(-1, 4000, (N,), device=DEV, generator=gen(N))
    want = cake.cake_kv_read(cache, slots)
    n = N * 3 * 96
    for by_head in (False, True):
        rooms = [torch.full((n + 32,), 7.0, dtype=BF16, device=DEV) for _ in range(2)]
        outs = [r[8:8 + n].view((3, N, 96) if by_head else (N, 3, 96)) for r in rooms]
        assert all(o.data_ptr() % 32 == 16 for o in outs)
        cake.cake_kv_read(cache, slots, out_k=outs[0], out_v=outs[1], by_head=by_head)
        for o, w, r in zip(outs, want, rooms):
            assert torch.equal(o.transpose(0, 1) if by_head else o, w)
            assert (r[:8] == 7).all() and (r[8 + n:] == 7).all()


def test_read_of_values_that_are_not_finite_slots_out_of_range_and_refusals():
    cache = cache_of(1, 4, 16, 2, 64, "e4m3", filled=True)
    cache.k.view(torch.uint8)[1, 3] = 0x7f
    ws = cake.alloc_append_workspace(DEV)
    slots = torch.tensor([19, 64, 2 ** 40, -5, 3, 3], device=DEV)
    k, v = cake.cake_kv_read(cache, slots, ws=ws)
    assert torch.isnan(k[0]).all() and (k[1:4] == 0).all() and (v[1:4] == 0).all() and torch.equal(k[4], k[5]) and (v[4] != 0).any()
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    assert cake.cake_kv_read(cache, slots[:0])[0].shape == (0, 2, 64)
    for bad in (dict(slots=slots.int()), dict(slots=slots[None]), dict(slots=slots[::2]), dict(out_k=torch.zeros(6, 2, 64, device=DEV)),
                dict(out_v=torch.zeros(2, 6, 64, dtype=BF16, device=DEV))):
        with pytest.raises(TypeError):
            cake.cake_kv_read(**{**dict(cache=cache, slots=slots), **bad})


def test_read_is_the_inverse_of_the_append():
    g = gen(7)
    T, Hkv, D = 500, 2, 128
    k, v = normal(g, T, Hkv, D), normal(g, T, Hkv, D)
    slots = torch.randperm(512, device=DEV, generator=g)[:T]
    cache = cache_of(1, 32, 16, Hkv, D, "bf16")
    cake.cake_kv_append(cache, k, v, slots)
    back = cake.cake_kv_read(cache, slots)
    assert torch.equal(back[0], k) and torch.equal(back[1], v)
    cache = cache_of(1, 32, 16, Hkv, D, "e4m3")
    cake.cake_kv_append(cache, k, v, slots)
    for got, want, sc in zip(cake.cake_kv_read(cache, slots), (k, v), (cache.k_scale, cache.v_scale)):
        clipped = want.double().clamp(-448 * sc.double()[None, :, None], 448 * sc.double()[None, :, None])
        bound = (2.0 ** -4 + 2.0 ** -8) * 1.01 * clipped.abs() + 2.0 ** -10 * 1.01 * sc.double()[None, :, None]
        close(got, clipped, bound, "back")
