"""The serving operators against plain implementations in 64 bits, at the sizes and masks where they can go wrong.

Tolerances, from the arithmetic alone (u = 2^-24 the rounding of fp32, half a unit in the last place: 2^-8 for bf16 (8 significant bits), 2^-4 for
e4m3, whose smallest step is 2^-9 of the scale):
  norm    s: one fp32 and one bf16 rounding, (2^-8 + 2^-23)|s|.  y: sum of H squares, rsqrt, two products: (H/2 + 8) u < 2e-3 relative
          for H <= 32768 in the worst case, so scale to 2e-3 at most (1e-5 asked for H <= 8192: errors of a sum in a tree),
          q within half a step of e4m3 of y / scale plus that
  gemm    fp32 accumulation in any order: (K + K/128 + 4) 2^-23 sum|terms| (2^-23: the tensor core may truncate), then the output's rounding
  append  three fp32 roundings of |a| + |b|, then the output's rounding
  decode  p held with 11 bits or more: 2^-11 sum p|v|; scores of D products: D 2^-23 sum|q k| scale, which moves p by as much;
          then the output's rounding
"""
import math

import pytest
import torch

import paper_2608_12629_b200 as cake

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
BF = 2.0 ** -8
U = 2.0 ** -23


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=BF16):
    return torch.empty(*shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def close(got, want, bound, what):
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound.clamp(min=1e-300)).max()):.3g} bounds"


# ------------------------------------------------------------------------------------------------------------- norm
def norm_ref(x, r, w, eps, norm=True):
    s = x.double() + (r.double() if r is not None else 0.0)
    y = s / (s.square().mean(1, keepdim=True) + eps).sqrt() if norm else s.clone()
    return s, y * w.double() if w is not None else y


def check_norm(x, r, w, group, q, scale, y, res, eps=1e-6, norm=True):
    T, H = x.shape
    s64, y64 = norm_ref(x, r, w, eps, norm)
    rel = 1e-5 if H <= 8192 else 2e-3
    if res is not None:
        close(res, s64, (BF + 2 * U) * s64.abs() + 1e-38, "residual")
    if y is not None:
        close(y, y64, (BF * 1.01 + rel) * y64.abs() + 1e-38, "y")
    if q is not None:
        g = group or H
        for i in range(scale.shape[1]):
            part = y64[:, i * g:(i + 1) * g]
            sc = (part.abs().amax(1) / 448.0).clamp(min=2.0 ** -100)
            close(scale[:, i], sc, rel * sc, "scale")
            own = scale[:, i].double()[:, None]
            close(q[:, i * g:(i + 1) * g].double() * own, part, (2.0 ** -4 + 2 * rel) * part.abs() + 2.0 ** -10 * 1.01 * own, "q")


@pytest.mark.parametrize("T,H,group,residual", [
    (1, 1, 128, True), (1, 8, 0, False), (3, 127, 128, True), (2, 128, 128, True), (5, 129, 0, True), (4, 136, 128, False),
    (7, 1000, 128, True), (1, 1023, 0, True), (2, 1025, 128, True), (9, 4096, 128, True), (3, 4104, 0, True), (2, 8191, 128, True),
    (2, 8200, 128, True), (1, 16384, 0, True), (2, 16392, 128, False), (1, 20001, 128, True), (1, 32768, 0, True), (1, 32767, 0, True),
    (1000, 64, 128, True), (257, 512, 0, False), (130, 5120, 128, True)])
def test_norm_shapes(T, H, group, residual):
    g = gen(T * 131 + H)
    x, w = normal(g, T, H, std=2.0), normal(g, H, std=0.3) + 1
    r = normal(g, T, H) if residual else None
    q, scale, y, res = cake.cake_rmsnorm_quant(x, w, r, group=group, want_y=True)
    assert (res is not None) == residual
    check_norm(x, r, w, group, q, scale, y, res)


@pytest.mark.parametrize("H,offset,stride", [(256, 0, 264), (256, 1, 300), (200, 0, 203), (1040, 8, 2080)])
def test_norm_strided_and_unaligned_rows(H, offset, stride):
    g = gen(H + offset)
    buf, rbuf = normal(g, 6, stride + offset + H), normal(g, 6, stride * 2 + H)
    x, r = buf[:, offset:offset + H], rbuf[:, 2:2 + H]
    q, scale, y, res = cake.cake_rmsnorm_quant(x, None, r, group=128, want_y=True)
    check_norm(x, r, None, 128, q, scale, y, res)


def test_norm_in_place_and_partial_outputs():
    g = gen(3)
    x, r, w = normal(g, 33, 768), normal(g, 33, 768), normal(g, 768) + 1
    x0, r0 = x.clone(), r.clone()
    q, scale, y, res = cake.cake_rmsnorm_quant(x, w, r, out_residual=r, out_y=x)
    assert res.data_ptr() == r.data_ptr() and y.data_ptr() == x.data_ptr()
    check_norm(x0, r0, w, 128, q, scale, y, res)
    q, scale, y, res = cake.cake_rmsnorm_quant(x0, w, want_q=False, want_y=True)
    assert q is None and scale is None and res is None
    check_norm(x0, None, w, 128, None, None, y, None)
    q, scale, y, res = cake.cake_rmsnorm_quant(x0, flags=cake.CAKE_RMSNORM_NONE, group=0)
    check_norm(x0, None, None, 0, q, scale, None, None, norm=False)


def test_norm_zero_rows_and_values_that_are_not_finite():
    x = torch.zeros(4, 256, dtype=BF16, device=DEV)
    x[1, 128:] = 3.0                                # a group of zeros beside one that is not
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    for group in (0, 128):
        q, scale, y, _ = cake.cake_rmsnorm_quant(x, group=group, want_y=True)
        assert (q[0].float() == 0).all() and (scale[0] == 2.0 ** -100).all()
        assert (q[1, :128].float() == 0).all() and torch.isfinite(q[1].float()).all()
        if group:
            assert scale[1, 0] == 2.0 ** -100
        assert torch.isnan(q[2, 5].float()) and torch.isnan(q[3].float()).all() and torch.isnan(y[3]).all()
    tiny = torch.full((1, 128), 2.0 ** -133, dtype=BF16, device=DEV)      # below the smallest scale's range
    q, scale, _, _ = cake.cake_rmsnorm_quant(tiny, flags=cake.CAKE_RMSNORM_NONE)
    assert torch.isfinite(q.float()).all() and (scale == 2.0 ** -100).all()


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("H,eps", [(256, 0.0), (256, 1e-30), (258, 1e-22), (257, 1e-30), (9000, 1e-30)])
def test_norm_rows_of_next_to_nothing_under_a_tiny_eps(H, eps, group):
    """1 / rms of 2^30 and more: the zeros among such a row's elements, and a row of zeros, stay zeros."""
    x = normal(gen(H), 5, H)
    x = (x.float() * torch.tensor([1.0, 2.0 ** -27, 2.0 ** -32, 2.0 ** -40, 0.0], device=DEV)[:, None]).to(BF16)
    x[:, :128] = 0.0                                 # a group of zeros
    if eps == 0.0:
        x = x[:4].contiguous()                       # (a row of zeros has no norm)
    w = normal(gen(1), H, std=0.3) + 1
    q, scale, y, _ = cake.cake_rmsnorm_quant(x, w, eps=eps, group=group, want_y=True)
    check_norm(x, None, w, group, q, scale, y, None, eps=eps)
    assert (q[:, :128].float() == 0).all()


def test_norm_no_rows_and_refusals():
    x = torch.zeros(0, 64, dtype=BF16, device=DEV)
    q, scale, _, _ = cake.cake_rmsnorm_quant(x)
    assert q.shape == (0, 64) and scale.shape == (0, 1)
    x = torch.zeros(2, 64, dtype=BF16, device=DEV)
    for bad, code in ((dict(group=64), cake.CAKE_ERR_UNSUPPORTED), (dict(flags=8), cake.CAKE_ERR_UNSUPPORTED),
                      (dict(want_q=False), cake.CAKE_ERR_NULL)):
        with pytest.raises(cake.CakeError) as e:
            cake.cake_rmsnorm_quant(x, **bad)
        assert e.value.code == code
    with pytest.raises(cake.CakeError) as e:
        cake.cake_rmsnorm_quant(torch.zeros(1, 32769, dtype=BF16, device=DEV))
    assert e.value.code == cake.CAKE_ERR_UNSUPPORTED
    for bad in (dict(weight=torch.zeros(63, dtype=BF16, device=DEV)), dict(out_q=torch.zeros(2, 64, dtype=torch.uint8, device=DEV))):
        with pytest.raises(TypeError):
            cake.cake_rmsnorm_quant(x, **bad)
    with pytest.raises(TypeError):
        cake.cake_rmsnorm_quant(x.float())
    with pytest.raises(ValueError):
        cake.cake_rmsnorm_quant(x, residual=x[:1])


# ------------------------------------------------------------------------------------------------------------- gemm
def gemm_inputs(M, N, K, seed):
    g = gen(seed)
    nk, nn = -(-K // 128), -(-N // 128)
    x, w = normal(g, M, K, std=60.0, dtype=E4M3), normal(g, N, K, std=60.0, dtype=E4M3)
    xs = torch.empty(M, nk, device=DEV).uniform_(1e-3, 2e-2, generator=g)
    ws = torch.empty(nn, nk, device=DEV).uniform_(1e-3, 2e-2, generator=g)
    return x, xs, w, ws


def check_gemm(x, xs, w, ws, out):
    M, K = x.shape
    N = w.shape[0]
    xd = x.double() * xs.double().repeat_interleave(128, 1)[:, :K]
    wd = w.double() * ws.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    want, size = xd @ wd.t(), xd.abs() @ wd.abs().t()
    step = BF * 1.01 if out.dtype == BF16 else U
    close(out, want, (K + K / 128 + 4) * U * size + step * want.abs() + 1e-30, "gemm")
    rel = float((out.double() - want).norm() / want.norm())
    assert rel <= (BF if out.dtype == BF16 else 1e-5), rel


@pytest.mark.parametrize("M", [1, 7, 16, 17, 32, 33, 64, 65, 128, 129, 200, 256, 300])
@pytest.mark.parametrize("N,K", [(1, 16), (127, 128), (128, 144), (129, 1040), (1000, 2048)])
def test_gemm_shapes(M, N, K):
    x, xs, w, ws = gemm_inputs(M, N, K, M + N + K)
    buf = cake.alloc_gemm_workspace(M, N, K, DEV)
    for dtype in (BF16, torch.float32):
        out = cake.cake_gemm_fp8(x, xs, w, ws, out_dtype=dtype, ws=buf)
        check_gemm(x, xs, w, ws, out)
    assert cake.cake_kmeans_device_status(buf) == cake.CAKE_OK


@pytest.mark.parametrize("M,N,K", [(3, 256, 12288), (700, 3001, 512), (2048, 2500, 1024), (1, 20000, 640), (160, 9216, 256)])
def test_gemm_many_tiles_and_long_contractions(M, N, K):
    """More tiles than SMs, several rounds of a persistent CTA, contractions that are split."""
    x, xs, w, ws = gemm_inputs(M, N, K, 5)
    buf = cake.alloc_gemm_workspace(M, N, K, DEV)
    a = cake.cake_gemm_fp8(x, xs, w, ws, out_dtype=torch.float32, ws=buf)
    check_gemm(x, xs, w, ws, a)
    for _ in range(3):                               # the same bits every time, from the same workspace
        assert torch.equal(cake.cake_gemm_fp8(x, xs, w, ws, out_dtype=torch.float32, ws=buf), a)
    assert cake.cake_kmeans_device_status(buf) == cake.CAKE_OK


def test_gemm_strides_and_one_workspace_for_many_sizes():
    big = cake.alloc_gemm_workspace(64, 4096, 8192, DEV)
    for M, N, K in [(64, 4096, 8192), (5, 200, 1024), (33, 1000, 4096), (64, 4096, 8192), (16, 128, 2048)]:
        x, xs, w, ws = gemm_inputs(M, N, K, M)
        xb = torch.zeros(M, K + 48, dtype=torch.uint8, device=DEV)
        xb.fill_(0x7f)                               # NaN around the rows
        xb[:, :K] = x.view(torch.uint8)
        wb = torch.full((N, K + 16), 0x7f, dtype=torch.uint8, device=DEV)
        wb[:, :K] = w.view(torch.uint8)
        need = cake.cake_gemm_fp8_workspace_bytes(M, N, K)
        assert need <= big.numel()
        out = torch.full((M, N + 3), 7.0, dtype=BF16, device=DEV)
        cake.cake_gemm_fp8(xb.view(E4M3)[:, :K], xs, wb.view(E4M3)[:, :K], ws, out=out[:, :N], ws=big)
        check_gemm(x, xs, w, ws, out[:, :N].contiguous())
        assert (out[:, N:] == 7.0).all()
    assert cake.cake_kmeans_device_status(big) == cake.CAKE_OK


def test_gemm_one_workspace_for_any_number_of_rows():
    """Plans with a split contraction and without one in turn, sizes that need less and more than the one before."""
    N, K = 1024, 4096
    buf = cake.alloc_gemm_workspace(None, N, K, DEV)
    assert len({cake.cake_gemm_fp8_workspace_bytes(m, N, K) for m in (4096, 300, 128, 64)}) > 2
    for M in (4096, 300, 128, 64, 1, 256, 5000, 65, 2048, 129):
        x, xs, w, ws = gemm_inputs(M, N, K, M)
        check_gemm(x, xs, w, ws, cake.cake_gemm_fp8(x, xs, w, ws, ws=buf))
    assert cake.cake_kmeans_device_status(buf) == cake.CAKE_OK


def test_gemm_integer_data_is_exact():
    """Small whole numbers, scales that are powers of two: every product and sum is exact, so a wrong block or row shows."""
    g = gen(9)
    M, N, K = 150, 300, 1152
    x = torch.randint(-8, 9, (M, K), generator=g, device=DEV).float().to(E4M3)
    w = torch.randint(-8, 9, (N, K), generator=g, device=DEV).float().to(E4M3)
    xs = 2.0 ** torch.randint(-2, 3, (M, 9), generator=g, device=DEV).float()
    ws = 2.0 ** torch.randint(-2, 3, (3, 9), generator=g, device=DEV).float()
    out = cake.cake_gemm_fp8(x, xs, w, ws, out_dtype=torch.float32)
    xd = x.double() * xs.double().repeat_interleave(128, 1)
    wd = w.double() * ws.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)
    assert torch.equal(out.double(), xd @ wd.t())


@pytest.mark.parametrize("M,N,K,parts", [
    (16, 128, 4096, 8), (3, 1920, 4096, 8), (3, 2048, 4096, 6), (16, 2816, 4096, 6), (16, 2944, 4096, 5), (33, 4224, 2048, 4),
    (33, 4352, 2048, 3), (1, 5760, 4096, 3), (1, 5888, 4096, 2), (64, 9472, 2048, 2), (64, 9600, 2048, 1), (5, 128, 384, 1)])
def test_gemm_order_of_sums_follows_from_the_sizes(M, N, K, parts):
    """Blocks of which each contributes its scale alone: fp32 sums of random numbers show in what order they were added.  The parts of a contraction
    (up to 64 rows) are those that the sizes say, whatever the device's SMs are grouped like."""
    nk = K // 128
    x, w = (torch.zeros(r, K, device=DEV) for r in (M, N))
    x[:, ::128] = 1.0
    w[:, ::128] = 1.0
    xs = torch.empty(M, nk, device=DEV).uniform_(0.1, 1.0, generator=gen(N))
    out = cake.cake_gemm_fp8(x.to(E4M3), xs, w.to(E4M3), torch.ones(N // 128, nk, device=DEV), out_dtype=torch.float32)
    want = torch.zeros(M, device=DEV)
    for s in range(parts):
        part = torch.zeros(M, device=DEV)
        for kb in range(s * nk // parts, (s + 1) * nk // parts):
            part = part + xs[:, kb]
        want = want + part
    assert torch.equal(out, want[:, None].expand(M, N))


def test_gemm_nan_stays_in_its_row_and_column():
    x, xs, w, ws = gemm_inputs(20, 140, 256, 1)
    x.view(torch.uint8)[3, 200] = 0x7f
    w.view(torch.uint8)[130, 5] = 0x7f
    out = cake.cake_gemm_fp8(x, xs, w, ws).float()
    bad = torch.isnan(out)
    assert bad[3].all() and bad[:, 130].all() and int(bad.sum()) == 140 + 20 - 1


def test_gemm_refusals():
    x, xs, w, ws = gemm_inputs(8, 32, 128, 2)
    assert cake.cake_gemm_fp8(x[:0], xs[:0], w, ws).shape == (0, 32)
    for M in (8, 200):
        x2, xs2, w2, ws2 = gemm_inputs(M, 128, 4096, 2)
        small = torch.zeros(cake.cake_gemm_fp8_workspace_bytes(M, 128, 4096) - 1, dtype=torch.uint8, device=DEV)
        with pytest.raises(cake.CakeError) as e:
            cake.cake_gemm_fp8(x2, xs2, w2, ws2, ws=small)
        assert e.value.code == cake.CAKE_ERR_WORKSPACE
    x3, xs3, w3, ws3 = gemm_inputs(8, 32, 120, 2)
    with pytest.raises(cake.CakeError) as e:
        cake.cake_gemm_fp8(x3, xs3, w3, ws3)
    assert e.value.code == cake.CAKE_ERR_ALIGN
    for bad in ((x, xs[:, :0], w, ws), (x, xs, w.view(torch.uint8), ws), (x, xs, w, ws.double())):
        with pytest.raises(TypeError):
            cake.cake_gemm_fp8(*bad)
    with pytest.raises(ValueError):
        cake.cake_gemm_fp8(x, xs, w[:, :112], ws)


# ----------------------------------------------------------------------------------------------------------- append
def rotary_table(n, rot):
    a = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    return torch.cat([a.cos(), a.sin()], 1).float()


def rotate_ref(x, pos, table, pairs):
    x = x.double().clone()
    mag = x.abs()
    if table is None:
        return x, mag
    rot = table.shape[1]
    c, s = table[pos.long()].double().chunk(2, 1)
    i = torch.arange(rot // 2, device=DEV)
    ia, ib = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
    a, b = x[:, :, ia], x[:, :, ib]
    x[:, :, ia], x[:, :, ib] = a * c[:, None] - b * s[:, None], b * c[:, None] + a * s[:, None]
    mag[:, :, ia] = mag[:, :, ib] = a.abs() + b.abs()
    return x, mag


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,pairs,page,kv,hnd", [
    (1, 1, 1, 64, 64, False, 1, BF16, False), (1, 8, 2, 128, 128, True, 16, BF16, True), (37, 32, 8, 128, 128, False, 16, BF16, False),
    (37, 32, 8, 128, 64, True, 16, E4M3, True), (50, 6, 3, 96, 48, False, 7, E4M3, False), (50, 6, 3, 96, 96, True, 100, BF16, False),
    (20, 4, 4, 256, 256, False, 64, E4M3, True), (20, 64, 1, 64, 32, False, 8, BF16, False), (33, 0, 2, 128, 128, False, 16, BF16, False),
    (33, 5, 1, 64, 0, False, 16, E4M3, False), (11, 3, 3, 64, 18, False, 4, BF16, False), (11, 3, 3, 64, 6, True, 4, E4M3, False),
    (300, 16, 16, 128, 128, False, 32, BF16, True)])
def test_append(T, Hq, Hkv, D, rot, pairs, page, kv, hnd):
    g = gen(T + Hq + D)
    pages = -(-2 * T // page) + 1
    shape = (pages, Hkv, page, D) if hnd else (pages, page, Hkv, D)
    kc, vc = (torch.full(shape, 0.5, device=DEV).to(kv) for _ in range(2))
    if hnd:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    ks = torch.empty(Hkv, device=DEV).uniform_(0.01, 0.1, generator=g) if kv == E4M3 else None
    vs = torch.empty(Hkv, device=DEV).uniform_(0.001, 0.1, generator=g) if kv == E4M3 else None      # some values saturate
    cache = cake.PagedCache(kc, vc, ks, vs)
    qkv = normal(g, T, Hq + 2 * Hkv, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    slots = torch.randperm(pages * page, device=DEV, generator=g)[:T].contiguous()
    slots[T // 2] = -1 if T > 2 else slots[T // 2]
    pos = torch.randint(0, 5000, (T,), device=DEV, generator=g, dtype=torch.int32)
    table = rotary_table(5000, rot) if rot else None
    ws = cake.alloc_append_workspace(DEV)
    before = [c.float().clone() for c in (kc, vc)]
    out = cake.cake_kv_append(cache, k, v, slots, pos if rot else None, table, q=q if Hq else None, interleaved=pairs, ws=ws)
    if Hq:
        want, mag = rotate_ref(q, pos, table, pairs)
        close(out, want, BF * 1.001 * want.abs() + 4 * U * mag + 1e-38, "q")
    else:
        assert out is None
    kept = slots >= 0
    for c, new, scale, old in ((kc, rotate_ref(k, pos, table, pairs), ks, before[0]), (vc, (v.double(), v.double().abs()), vs, before[1])):
        want, mag = new
        got = c.float()[slots[kept] // page, slots[kept] % page]
        sc = scale.double()[None, :, None] if scale is not None else 1.0
        held = (want / sc).clamp(-448, 448) if scale is not None else want
        step = 2.0 ** -4 if kv == E4M3 else BF * 1.001
        close(got, held[kept], (step * held.abs() + 4 * U * mag / sc)[kept] + (2.0 ** -10 if kv == E4M3 else 1e-38), "cache")
        rest = torch.ones(pages, page, dtype=torch.bool, device=DEV)
        rest[slots[kept] // page, slots[kept] % page] = False
        assert torch.equal(c.float()[rest], old[rest])
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


def test_append_places_that_do_not_exist():
    g = gen(4)
    kc, vc = (torch.zeros(4, 8, 2, 64, dtype=BF16, device=DEV) for _ in range(2))
    cache = cake.PagedCache(kc, vc)
    k, v, q = normal(g, 4, 2, 64), normal(g, 4, 2, 64), normal(g, 4, 4, 64)
    ws = cake.alloc_append_workspace(DEV)
    table = rotary_table(16, 64)
    out = torch.full((4, 4, 64), 9.0, dtype=BF16, device=DEV)
    slots = torch.tensor([0, 32, 2 ** 40, 5], device=DEV)
    pos = torch.tensor([3, 3, 3, 16], dtype=torch.int32, device=DEV)
    cake.cake_kv_append(cache, k, v, slots, pos, table, q=q, out_q=out, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK
    assert (vc.view(-1, 2, 64)[0] == v[0]).all() and (vc.view(-1, 2, 64)[1:] == 0).all() and (kc.view(-1, 2, 64)[1:] == 0).all()
    want, mag = rotate_ref(q[:3], pos[:3], table, False)
    close(out[:3], want, BF * 1.001 * want.abs() + 4 * U * mag, "q")
    assert (out[3] == 9.0).all()                     # a position without a row in the table: nothing of the token is written


@pytest.mark.parametrize("pairs", [False, True])
def test_append_unaligned_sources(pairs):
    """Keys, values and queries at odd addresses and strides: the element-wise kernel, against the wide one bit for bit."""
    g = gen(8)
    T, Hq, Hkv, D = 9, 3, 2, 128
    q, k, v = normal(g, T, Hq, D), normal(g, T, Hkv, D), normal(g, T, Hkv, D)
    slots, pos, table = torch.arange(T, device=DEV), torch.arange(T, dtype=torch.int32, device=DEV) * 7, rotary_table(64, 64)
    caches = [[torch.zeros(2, 8, Hkv, D, dtype=kv, device=DEV) for _ in range(2)] for kv in (BF16, BF16)]
    outs = []
    for i, c in enumerate(caches):
        args = (k, v, q)
        if i:
            args = []
            for t in (k, v, q):
                buf = torch.zeros(T * (t[0].numel() + 1) + 1, dtype=BF16, device=DEV)
                odd = torch.as_strided(buf, t.shape, (t[0].numel() + 1, D, 1), 1)
                odd.copy_(t)
                args.append(odd)
        outs.append(cake.cake_kv_append(cake.PagedCache(*c), args[0], args[1], slots, pos, table, q=args[2], interleaved=pairs))
    assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("kv", [BF16, E4M3])
def test_append_bits_do_not_depend_on_alignment(kv, pairs):
    T, Hq, Hkv, D, rot = 300, 8, 4, 128, 64
    g = gen(31)
    q, k, v = normal(g, T, Hq, D), normal(g, T, Hkv, D), normal(g, T, Hkv, D)
    ang = torch.empty(500, rot // 2, device=DEV).uniform_(0, 6.28, generator=g)
    table = torch.cat([ang.cos(), ang.sin()], 1).contiguous()
    pos = torch.randint(0, 500, (T,), generator=g, device=DEV, dtype=torch.int32)
    slots = torch.randperm(20 * 16, generator=g, device=DEV)[:T]
    ks, vs = torch.empty(2, Hkv, device=DEV).uniform_(0.001, 0.02, generator=g)

    def odd(t):                                       # the same elements, two bytes off
        room = torch.empty(t.numel() + 1, dtype=BF16, device=DEV)
        room[1:] = t.flatten()
        return room[1:].view(t.shape)

    results = []
    for change in (lambda t: t, odd):
        kc, vc = (torch.zeros(20, 16, Hkv, D, dtype=kv, device=DEV) for _ in range(2))
        cache = cake.PagedCache(kc, vc, ks, vs) if kv == E4M3 else cake.PagedCache(kc, vc)
        out = cake.cake_kv_append(cache, change(k), change(v), slots, pos, table, change(q), interleaved=pairs)
        results.append((out, kc.view(torch.uint8), vc.view(torch.uint8)))
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [20, 3000])
def test_append_a_slot_named_twice(T):
    """Its elements are of the one or the other token; every other slot is what it would be without the second."""
    g = gen(T)
    Hkv, D, page = 3, 64, 16
    k, v = normal(g, T, Hkv, D), normal(g, T, Hkv, D)
    slots = torch.randperm(2 * T, generator=g, device=DEV)[:T]
    twin = torch.randperm(T, generator=g, device=DEV)[:T // 4 * 2].view(2, -1)
    slots[twin[1]] = slots[twin[0]]
    kc, vc = (torch.full((-(-2 * T // page), page, Hkv, D), 7.0, dtype=BF16, device=DEV) for _ in range(2))
    cake.cake_kv_append(cake.PagedCache(kc, vc), k, v, slots)
    for cache, new in ((kc, k), (vc, v)):
        flat = cache.view(-1, Hkv, D)
        here = flat[slots[twin[0]]]
        assert ((here == new[twin[0]]) | (here == new[twin[1]])).all()
        once = torch.ones(T, dtype=torch.bool, device=DEV)
        once[twin.flatten()] = False
        assert torch.equal(flat[slots[once]], new[once])
        rest = torch.ones(flat.shape[0], dtype=torch.bool, device=DEV)
        rest[slots] = False
        assert (flat[rest] == 7.0).all()


def test_append_in_place_queries_and_refusals():
    g = gen(6)
    kc = torch.zeros(4, 8, 2, 128, dtype=BF16, device=DEV)
    cache = cake.PagedCache(kc, kc.clone())
    q, k, v = normal(g, 5, 4, 128), normal(g, 5, 2, 128), normal(g, 5, 2, 128)
    slots, pos, table = torch.arange(5, device=DEV), torch.arange(5, dtype=torch.int32, device=DEV), rotary_table(8, 128)
    for pairs in (False, True):
        mine = q.clone()
        want, mag = rotate_ref(q, pos, table, pairs)
        assert cake.cake_kv_append(cache, k, v, slots, pos, table, q=mine, out_q=mine, interleaved=pairs).data_ptr() == mine.data_ptr()
        close(mine, want, BF * 1.001 * want.abs() + 4 * U * mag, "q in place")
    with pytest.raises(ValueError):
        cake.cake_kv_append(cache, k[:, :1], v[:, :1], slots)
    with pytest.raises(TypeError):
        cake.cake_kv_append(cache, k, v, slots.int())
    with pytest.raises(TypeError):
        cake.cake_kv_append(cache, k, v, slots, pos, table.double())
    with pytest.raises(ValueError):
        cake.cake_kv_append(cache, k, v, slots, None, table)
    with pytest.raises(cake.CakeError) as e:
        cake.cake_kv_append(cache, k, v, slots, pos, table[:, :127].contiguous())
    assert e.value.code == cake.CAKE_ERR_SHAPE
    with pytest.raises(cake.CakeError) as e:
        cake.cake_kv_append(cache, k, v, slots, ws=torch.zeros(256, dtype=torch.uint8, device=DEV))
    assert e.value.code == cake.CAKE_ERR_WORKSPACE
    odd = torch.zeros(4, 8, 2, 80, dtype=BF16, device=DEV)
    with pytest.raises(cake.CakeError) as e:
        cake.cake_kv_append(cake.PagedCache(odd, odd), k[..., :80].contiguous(), v[..., :80].contiguous(), slots)
    assert e.value.code == cake.CAKE_ERR_UNSUPPORTED
    off = torch.zeros(4 * 8 * 2 * 64 + 4, dtype=BF16, device=DEV)[4:].view(4, 8, 2, 64)
    with pytest.raises(cake.CakeError) as e:
        cake.cake_kv_append(cake.PagedCache(off, off), k[..., :64].contiguous(), v[..., :64].contiguous(), slots)
    assert e.value.code == cake.CAKE_ERR_ALIGN
    assert cake.cake_kv_append(cache, k[:0], v[:0], slots[:0]) is None


# ----------------------------------------------------------------------------------------------------------- decode
def decode_problem(Hq, Hkv, D, page, kv, lens, seed, per_head=False, hnd=False, poison=True, std=1.0):
    """A cache whose tokens behind every length, and whose unused pages, hold NaN; table entries behind the last page are invalid."""
    g = gen(seed)
    lens = torch.tensor(lens, dtype=torch.int32).view(len(lens), -1)
    B = lens.shape[0]
    need = -(-lens // page)
    width = max(1, int(need.max()))
    rows = lens.shape[1]
    pages = int(need.sum()) + 2
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))
    table = torch.full((B, rows, width), 2 ** 30, dtype=torch.int32)
    shape = (pages, Hkv, page, D) if hnd else (pages, page, Hkv, D)
    e = kv == E4M3
    kc, vc = (normal(g, *shape, std=60.0 if e else std, dtype=kv) for _ in range(2))
    if hnd:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    used = torch.zeros(pages, page, Hkv, dtype=torch.bool)
    at = 0
    for b in range(B):
        for r in range(rows):
            n, L = int(need[b, r]), int(lens[b, r])
            mine = order[at:at + n]
            at += n
            table[b, r, :n] = mine.int()
            tok = torch.arange(L)
            if per_head:
                used[mine[tok // page], tok % page, r] = True
            else:
                used[mine[tok // page], tok % page] = True
    if poison:
        for c in (kc, vc):
            raw = c.view(torch.uint8) if e else c
            raw[~used.to(DEV)] = 0x7f if e else float("nan")
    ks = torch.empty(Hkv, device=DEV).uniform_(0.01, 0.03, generator=g) if e else None
    vs = torch.empty(Hkv, device=DEV).uniform_(0.01, 0.03, generator=g) if e else None
    q = normal(g, B, Hq, D, std=1.5)
    if not per_head:
        table, lens = table[:, 0], lens[:, 0]
    return q, cake.PagedCache(kc, vc, ks, vs), table.contiguous().to(DEV), lens.contiguous().to(DEV)


def check_decode(q, cache, table, lens, out, lse, window=0, scale=None):
    B, Hq, D = q.shape
    Hkv, page = cache.Hkv, cache.page_size
    G = Hq // Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    for b in range(B):
        for h in range(Hkv):
            n = int(lens[b, h] if lens.dim() == 2 else lens[b])
            a = max(0, n - window) if window else 0
            rows = slice(h * G, (h + 1) * G)
            if n - a <= 0:
                assert (out[b, rows] == 0).all() and (lse is None or (lse[b, rows] == -math.inf).all())
                continue
            t = (table[b, h] if table.dim() == 3 else table[b])[:-(-n // page)].long()
            k = cache.k[t, :, h].reshape(-1, D)[a:n].double() if cache.k.dtype == BF16 else cache.k.float()[t, :, h].reshape(-1, D)[a:n].double()
            v = cache.v[t, :, h].reshape(-1, D)[a:n].double() if cache.v.dtype == BF16 else cache.v.float()[t, :, h].reshape(-1, D)[a:n].double()
            if cache.k_scale is not None:
                k, v = k * cache.k_scale[h].double(), v * cache.v_scale[h].double()
            qq = q[b, rows].double()
            x = qq @ k.t() * scale
            p = torch.softmax(x, 1)
            want, size = p @ v, p @ v.abs()
            dx = (D * U * (qq.abs() @ k.abs().t()) * scale).amax(1, keepdim=True) + 4 * U * x.abs().amax(1, keepdim=True)
            close(out[b, rows], want, BF * 1.001 * want.abs() + (2.0 ** -11 + 4 * dx) * size + 1e-30, f"out {b},{h}")
            if lse is not None:
                ref = torch.logsumexp(x, 1)
                close(lse[b, rows], ref, dx[:, 0] + 1e-5 + 4 * U * ref.abs() + n * U, f"lse {b},{h}")


CASES = [
    # Hq, Hkv, D, page, kv, lens, window
    (1, 1, 64, 1, BF16, [1], 0), (8, 1, 64, 16, BF16, [0], 0), (4, 2, 128, 16, BF16, [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129], 0),
    (32, 8, 128, 16, BF16, [777], 0), (8, 8, 96, 7, BF16, [100, 3, 0, 250], 0), (12, 4, 96, 100, E4M3, [100, 3, 0, 250, 1000], 0),
    (16, 1, 128, 64, E4M3, [300, 1], 0), (9, 1, 128, 32, BF16, [500], 0), (24, 1, 64, 16, BF16, [400, 77], 0),
    (40, 1, 256, 16, BF16, [90, 200], 0), (8, 8, 256, 8, E4M3, [33, 64], 0), (16, 1, 256, 16, E4M3, [1000], 0),
    (2, 2, 64, 1, E4M3, [5, 130, 64], 0), (5, 1, 64, 16, BF16, [3000], 100), (8, 2, 128, 16, E4M3, [50, 64, 65, 1000], 64),
    (4, 1, 128, 48, BF16, [200, 10], 1), (64, 8, 128, 64, E4M3, [2000, 1], 0), (2, 1, 128, 16, BF16, [20000], 0),
    (6, 2, 64, 16, BF16, [9000, 0, 1, 4000], 0)]


@pytest.mark.parametrize("Hq,Hkv,D,page,kv,lens,window", CASES)
@pytest.mark.parametrize("hnd", [False, True])
def test_decode_shapes(Hq, Hkv, D, page, kv, lens, window, hnd):
    q, cache, table, n = decode_problem(Hq, Hkv, D, page, kv, lens, Hq + D + len(lens), hnd=hnd)
    ws = cake.alloc_decode_workspace(len(lens), Hq, Hkv, D, DEV)
    out, lse = cake.cake_paged_decode(q, cache, table, n, window=window, want_lse=True, ws=ws)
    check_decode(q, cache, table, n, out, lse, window)
    again, none = cake.cake_paged_decode(q, cache, table, n, window=window, ws=ws)
    assert none is None and torch.equal(again, out)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


@pytest.mark.parametrize("Hq,Hkv,D,page,kv", [(16, 16, 64, 1, BF16), (8, 4, 128, 1, E4M3), (6, 3, 128, 16, BF16)])
def test_decode_a_table_per_head(Hq, Hkv, D, page, kv):
    lens = [[(37 * i * (h + 1)) % 411 for h in range(Hkv)] for i in range(3)]
    q, cache, table, n = decode_problem(Hq, Hkv, D, page, kv, lens, 8, per_head=True)
    out, lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True)
    check_decode(q, cache, table, n, out, lse)


def test_decode_many_sequences_and_one_workspace_for_many_shapes():
    ws = cake.alloc_decode_workspace(1, 32, 1, 256, DEV)          # the largest of the shapes below
    for B, Hq, Hkv, D in [(300, 4, 2, 64), (1, 32, 1, 256), (129, 8, 8, 128), (2, 2, 1, 64), (700, 1, 1, 128)]:
        lens = [(i * 53) % 190 if B > 2 else 5000 for i in range(B)]
        q, cache, table, n = decode_problem(Hq, Hkv, D, 16, BF16, lens, B)
        assert cake.cake_paged_decode_workspace_bytes(B, Hq, Hkv, D) <= ws.numel()
        out, lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True, ws=ws)
        check_decode(q, cache, table, n, out, lse)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


@pytest.mark.parametrize("B,Hq,Hkv,D,kv,length", [(1, 16, 1, 256, BF16, 30000), (2, 6, 1, 128, E4M3, 40000), (1, 20, 1, 96, BF16, 20000),
                                                  (1, 3, 1, 64, BF16, 70001), (3, 40, 2, 64, E4M3, 9000)])
def test_decode_few_sequences_in_many_parts(B, Hq, Hkv, D, kv, length):
    """Rows split over hundreds of CTAs (the parts are joined by a kernel of their own), between calls that are not split."""
    ws = cake.alloc_decode_workspace(B, Hq, Hkv, D, DEV)
    for lens in ([length] * B, [7] * B, [length - 11 * i for i in range(B)], [0] * B, [length // (i + 1) for i in range(B)]):
        q, cache, table, n = decode_problem(Hq, Hkv, D, 16, kv, lens, length)
        wide = torch.full((B, -(-length // 16)), -1, dtype=torch.int32, device=DEV)      # the table's width says how long rows may be
        wide[:, :table.shape[1]] = table
        out, lse = cake.cake_paged_decode(q, cache, wide, n, want_lse=True, ws=ws)
        check_decode(q, cache, table, n, out, lse)
        assert torch.equal(cake.cake_paged_decode(q, cache, wide, n, ws=ws)[0], out)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


@pytest.mark.parametrize("Hq,Hkv,D,lens,width,window", [
    (32, 8, 128, [777], 1024, 0),                    # a table with room for 16,384 tokens
    (4, 1, 128, [5], 8192, 0), (16, 1, 64, [16000], 1024, 100), (64, 8, 128, [16000, 300], 1024, 300), (16, 1, 256, [30000], 1875, 60)])
def test_decode_short_rows_take_one_launch_whatever_the_table_has_room_for(Hq, Hkv, D, lens, width, window):
    q, cache, table, n = decode_problem(Hq, Hkv, D, 16, BF16, lens, 41)
    wide = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    ws = cake.alloc_decode_workspace(len(lens), Hq, Hkv, D, DEV)
    before = cake.cake_kmeans_kernel_launches()
    out, lse = cake.cake_paged_decode(q, cache, wide, n, window=window, want_lse=True, ws=ws)
    assert cake.cake_kmeans_kernel_launches() == before + 1
    check_decode(q, cache, table, n, out, lse, window)


@pytest.mark.parametrize("Hq,Hkv,D,kv,page,lens,window", [
    (4, 1, 128, BF16, 16, [40000], 0),               # 444 parts in two levels: one row
    (8, 2, 64, E4M3, 16, [30000, 11], 0),            # a CTA ends one row's last group and begins the next's first
    (3, 1, 128, BF16, 7, [9000, 20001, 5], 9500),    # and a window
    (16, 1, 256, BF16, 16, [30000] + [40] * 149, 0), (32, 2, 128, E4M3, 32, [5] * 80 + [60000] + [90] * 79, 0),
    (12, 1, 96, BF16, 16, [17] * 199 + [25000], 20000), (20, 1, 64, E4M3, 16, [30000] * 2 + [1] * 160, 0)])
def test_decode_rows_of_many_parts_joined_in_two_levels(Hq, Hkv, D, kv, page, lens, window):
    """Long rows, alone or beside many short ones, that no second kernel joins: between calls of other lengths in the same workspace."""
    ws = cake.alloc_decode_workspace(len(lens), Hq, Hkv, D, DEV)
    for change in (lambda x: x, lambda x: [min(n, 50) for n in x], lambda x: x[::-1], lambda x: [n // 3 for n in x], lambda x: x):
        q, cache, table, n = decode_problem(Hq, Hkv, D, page, kv, change(lens), 43)
        before = cake.cake_kmeans_kernel_launches()
        out, lse = cake.cake_paged_decode(q, cache, table, n, window=window, want_lse=True, ws=ws)
        assert cake.cake_kmeans_kernel_launches() == before + 1
        check_decode(q, cache, table, n, out, lse, window)
        for _ in range(3):
            assert torch.equal(cake.cake_paged_decode(q, cache, table, n, window=window, ws=ws)[0], out)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


@pytest.mark.parametrize("Hq,Hkv,D,kv,lens,window", [
    (16, 1, 128, BF16, [30000], 9000), (32, 2, 64, E4M3, [[20000, 9], [0, 12345]], 0), (32, 2, 256, BF16, [[15000, 4000]], 5001),
    (6, 2, 128, E4M3, [[8000, 30000]], 0), (4, 4, 64, BF16, [[500, 0, 20000, 64]] * 3, 333)])
def test_decode_windows_and_tables_per_head_in_many_parts(Hq, Hkv, D, kv, lens, window):
    """The join's kernel, and two levels, with windows and with lengths and tables per head."""
    per_head = isinstance(lens[0], list)
    page = 1 if D == 64 else 16
    q, cache, table, n = decode_problem(Hq, Hkv, D, page, kv, lens, 47, per_head=per_head)
    ws = cake.alloc_decode_workspace(len(lens), Hq, Hkv, D, DEV)
    for w in (window, 0, 17):
        out, lse = cake.cake_paged_decode(q, cache, table, n, window=w, want_lse=True, ws=ws)
        check_decode(q, cache, table, n, out, lse, w)
        assert torch.equal(cake.cake_paged_decode(q, cache, table, n, window=w, ws=ws)[0], out)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


def test_decode_scores_far_apart_and_infinite():
    """A maximum that arrives late, scores of -inf beside finite ones, and a row that is nothing but -inf or NaN."""
    q, cache, table, n = decode_problem(8, 1, 64, 16, BF16, [600, 600, 200, 200], 3, poison=False)
    q[:, :, 0] = 1.0
    cache.k[..., 0] = 0.0
    slot = lambda b, t: (int(table[b, t // 16]), t % 16)  # noqa: E731
    p, o = slot(0, 599)
    cache.k[p, o, 0, 0] = 2000.0                     # one token outweighs all before it
    for t in range(0, 600, 2):
        p, o = slot(1, t)
        cache.k[p, o, 0, 0] = -math.inf              # half of the tokens weigh nothing
    for t in range(200):
        p, o = slot(2, t)
        cache.k[p, o, 0, 0] = -math.inf
    p, o = slot(3, 50)
    cache.k[p, o, 0, 0] = math.nan
    out, lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True)
    check_decode(q[:1], cache, table[:1], n[:1], out[:1], lse[:1])
    idx = torch.arange(1, 600, 2, device=DEV)
    k = cache.k[table[1].long()].reshape(-1, 64)[idx].double()
    v = cache.v[table[1].long()].reshape(-1, 64)[idx].double()
    x = q[1].double() @ k.t() / 8
    want, size = torch.softmax(x, 1) @ v, torch.softmax(x, 1) @ v.abs()
    close(out[1], want, BF * 1.001 * want.abs() + 2.0 ** -10 * size, "half weighs nothing")
    assert (out[2] == 0).all() and (lse[2] == -math.inf).all()
    assert torch.isnan(out[3]).all() and torch.isnan(lse[3]).all()


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_decode_every_8_bit_value_and_nan(D):
    """All 254 finite e4m3 patterns (their subnormals too) through the keys' and the values' conversion; NaN where it is."""
    q, cache, table, n = decode_problem(4, 1, D, 16, E4M3, [256, 256, 256], 21, poison=False)
    flat = [c.view(torch.uint8) for c in (cache.k, cache.v)]
    codes = torch.arange(256, device=DEV)
    codes = torch.where((codes & 0x7f) == 0x7f, codes - 1, codes).to(torch.uint8)
    g = gen(2)
    for b in range(3):
        for f in flat:                               # every token of a column another code
            cols = torch.stack([codes[torch.randperm(256, device=DEV, generator=g)] for _ in range(D)], 1)
            f[table[b].long()] = cols.view(16, 16, 1, D)
    q.mul_(0.02)
    out, lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True)
    check_decode(q, cache, table, n, out, lse)
    for sign in (0x7f, 0xff):
        flat[0][table[0, 3].long(), 5, 0, 7] = sign  # a key of the first sequence
        flat[1][table[1, 9].long(), 2, 0, D - 1] = sign      # one element of a value of the second
        bad, bad_lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True)
        assert torch.isnan(bad[0]).all() and torch.isnan(bad_lse[0]).all()
        assert torch.isnan(bad[1, :, D - 1]).all() and torch.equal(bad[1, :, :D - 1], out[1, :, :D - 1])
        assert torch.equal(bad[2], out[2]) and torch.equal(bad_lse[1:], lse[1:])


@pytest.mark.parametrize("kv", [BF16, E4M3])
@pytest.mark.parametrize("D,G", [(64, 1), (96, 4), (128, 12), (256, 2)])
@pytest.mark.parametrize("gap", [14.3, 25.5, 28.7, 31.0])
def test_decode_many_light_weights_beside_a_heavy_one(gap, D, G, kv):
    """Weights 2^-gap of the heaviest, thousands of them, and nothing else in the output.  A weight is held with 11 bits, or to 2^-36 of the
    heaviest where that is more; scores of up to 31 are right to 32 * 2^-22; then the output's rounding."""
    B, N, page = 640, 2048, 32
    k = torch.zeros(N // page, page, 1, D, dtype=torch.float32, device=DEV)
    v = torch.ones_like(k)
    flat_k, flat_v = k.view(N, D), v.view(N, D)
    flat_k[0:64:16, 0] = 1.0                          # one in every 16 keys of the first 64, of value zero
    flat_v[0:64:16] = 0.0
    cache = cake.PagedCache(k.to(kv), v.to(kv))
    q = torch.zeros(B, G, D, dtype=BF16, device=DEV)
    q[:, :, 0] = 1.0
    table = torch.arange(N // page, dtype=torch.int32, device=DEV)[None].expand(B, -1).contiguous()
    n = torch.full((B,), N, dtype=torch.int32, device=DEV)
    scale = torch.tensor(gap * math.log(2.0), dtype=torch.float32).item()
    out, _ = cake.cake_paged_decode(q, cache, table, n, scale=scale)
    p = math.exp(-scale)
    want = (N - 4) * p / (4 + (N - 4) * p)
    rel = BF + max(2.0 ** -11, 2.0 ** -36 / p) + 32 * 2.0 ** -22 + N * U
    close(out, torch.full_like(out, want, dtype=torch.float64), torch.full_like(out, rel * want, dtype=torch.float64), "out")


def test_decode_scale_strides_streams_and_graphs():
    q, cache, table, n = decode_problem(8, 2, 128, 16, BF16, [500, 33, 0, 70], 12)
    wide = torch.zeros(4, 12, 128, dtype=BF16, device=DEV)
    wide[:, 2:10] = q
    out, lse = cake.cake_paged_decode(wide[:, 2:10], cache, table, n, scale=0.3, want_lse=True)
    check_decode(q, cache, table, n, out, lse, scale=0.3)
    big = torch.full((4, table.shape[1] + 5), -7, dtype=torch.int32, device=DEV)
    big[:, :table.shape[1]] = table
    side = torch.cuda.Stream()
    ws = cake.alloc_decode_workspace(4, 8, 2, 128, DEV)
    mine = torch.empty_like(out)
    side.wait_stream(torch.cuda.current_stream())
    cake.cake_paged_decode(q, cache, big[:, :table.shape[1]], n, scale=0.3, out=mine, ws=ws, stream=side)
    side.synchronize()
    assert torch.equal(mine, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cake.cake_paged_decode(q, cache, table, n, scale=0.3, out=mine, ws=ws)
    n[2] = 40                                        # lengths are read when the graph runs
    table[2, :3] = table[0, :3]
    mine.zero_()
    graph.replay()
    torch.cuda.synchronize()
    check_decode(q, cache, table, n, mine, None, scale=0.3)


@pytest.mark.parametrize("kv", [BF16, E4M3])
def test_decode_unaligned_queries_and_output(kv):
    """Queries and output on odd addresses take element-wise accesses; a table of no pages leaves every row empty."""
    q, cache, table, n = decode_problem(6, 2, 128, 16, kv, [90, 0, 300], 31)
    buf = torch.zeros(3 * 7 * 129 + 1, dtype=BF16, device=DEV)
    odd = torch.as_strided(buf, (3, 6, 128), (7 * 129, 129, 1), 1)
    odd.copy_(q)
    out = torch.zeros(q.numel() + 1, dtype=BF16, device=DEV)[1:].view(q.shape)
    want, _ = cake.cake_paged_decode(q, cache, table, n)
    cake.cake_paged_decode(odd, cache, table, n, out=out)
    assert torch.equal(out, want)
    none, lse = cake.cake_paged_decode(q, cache, table[:, :0], torch.zeros_like(n), want_lse=True)
    assert (none == 0).all() and (lse == -math.inf).all()


def test_decode_pages_that_do_not_exist():
    q, cache, table, n = decode_problem(4, 1, 64, 16, BF16, [100], 5)
    ws = cake.alloc_decode_workspace(1, 4, 1, 64, DEV)
    bad = table.clone()
    bad[0, 2], bad[0, 5] = -1, cache.num_pages
    out, lse = cake.cake_paged_decode(q, cache, bad, n, want_lse=True, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    keep = torch.cat([table[0, :2], table[0, 3:5], table[0, 6:7]])[None].contiguous()
    want, want_lse = cake.cake_paged_decode(q, cache, keep, n - 32, want_lse=True)
    assert torch.allclose(out.float(), want.float(), atol=2e-2) and torch.allclose(lse, want_lse, atol=1e-4)
    out, lse = cake.cake_paged_decode(q, cache, torch.full_like(table, -1), n, want_lse=True, ws=ws)
    assert (out == 0).all() and (lse == -math.inf).all()
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    out, _ = cake.cake_paged_decode(q, cache, table[:, :2].contiguous(), n, ws=ws)       # a length beyond the table is cut
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    check_decode(q, cache, table, torch.tensor([32], dtype=torch.int32, device=DEV), out, None)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes (and 2^31 elements) per side: tokens in its last pages."""
    pages, page, D = 2 ** 20 + 9, 16, 128
    kc, vc = (torch.empty(pages, page, 1, D, dtype=BF16, device=DEV) for _ in range(2))
    cache = cake.PagedCache(kc, vc)
    g = gen(1)
    T = 70
    k, v = normal(g, T, 1, D), normal(g, T, 1, D)
    slots = (pages * page - 5 * page + torch.arange(T, device=DEV))
    cake.cake_kv_append(cache, k, v, slots)
    table = torch.arange(pages - 5, pages, dtype=torch.int32, device=DEV)[None].contiguous()
    n = torch.tensor([T], dtype=torch.int32, device=DEV)
    q = normal(g, 1, 4, D)
    assert torch.equal(kc.view(-1, D)[slots], k[:, 0]) and torch.equal(vc.view(-1, D)[slots], v[:, 0])
    out, lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True)
    check_decode(q, cache, table, n, out, lse)


def test_strides_of_single_elements_say_nothing():
    """One page, one head: their strides may be any number, one that is no multiple of 16 bytes too."""
    g = gen(8)
    room_k, room_v = normal(g, 16 * 64 + 9), normal(g, 16 * 64 + 9)
    k, v = (torch.as_strided(t, (1, 16, 1, 64), (1033, 64, 13, 1)) for t in (room_k, room_v))
    plain = cake.PagedCache(k.contiguous(), v.contiguous())
    cache = cake.PagedCache(k, v)
    q = normal(g, 1, 1, 64)
    table, n = torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.tensor([11], dtype=torch.int32, device=DEV)
    out, lse = cake.cake_paged_decode(torch.as_strided(q, (1, 1, 64), (77, 3, 1)), cache, table, n, want_lse=True)
    check_decode(q, plain, table, n, out, lse)
    new_k, new_v = normal(g, 1, 1, 64), normal(g, 1, 1, 64)
    cake.cake_kv_append(cache, new_k, new_v, torch.tensor([15], dtype=torch.int64, device=DEV))
    assert torch.equal(k[0, 15], new_k[0]) and torch.equal(v[0, 15], new_v[0])


def test_decode_refusals():
    q, cache, table, n = decode_problem(4, 2, 64, 16, BF16, [20], 5)
    assert cake.cake_paged_decode(q[:0], cache, table[:0], n[:0])[0].shape == (0, 4, 64)
    for bad in (dict(q=q.float()), dict(table=table.long()), dict(n=n.long())):
        with pytest.raises(TypeError):
            cake.cake_paged_decode(bad.get("q", q), cache, bad.get("table", table), bad.get("n", n))
    with pytest.raises(ValueError):
        cake.cake_paged_decode(q, cache, table, torch.cat([n, n]))
    with pytest.raises(cake.CakeError) as e:
        cake.cake_paged_decode(q[:, :3].contiguous(), cache, table, n)
    assert e.value.code == cake.CAKE_ERR_SHAPE
    with pytest.raises(cake.CakeError) as e:
        cake.cake_paged_decode(q, cache, table, n, window=-1)
    assert e.value.code == cake.CAKE_ERR_SHAPE
    with pytest.raises(cake.CakeError) as e:
        cake.cake_paged_decode(q, cache, table, n, ws=torch.zeros(cake.CAKE_SERVING_HEADER_BYTES, dtype=torch.uint8, device=DEV))
    assert e.value.code == cake.CAKE_ERR_WORKSPACE


def test_scratch_and_outputs_of_another_stream():
    """Calls on a stream that is not the current one: what they allocate is zeroed on theirs and stays theirs until their kernels are done,
    whatever the current stream does meanwhile with the memory it frees."""
    g = gen(77)
    q, cache, table, n = decode_problem(32, 8, 128, 16, BF16, [3000, 17], 4)
    x, w = normal(g, 70, 1024), normal(g, 1024)
    X, xs, W, wsc = gemm_inputs(100, 256, 4096, 5)
    k, v, slots = normal(g, 9, 8, 128), normal(g, 9, 8, 128), torch.arange(9, dtype=torch.int64, device=DEV)
    qs = normal(g, 9, 32, 128)
    spare = cake.PagedCache(torch.zeros(4, 16, 8, 128, dtype=BF16, device=DEV), torch.zeros(4, 16, 8, 128, dtype=BF16, device=DEV))

    def run(stream):
        a = cake.cake_rmsnorm_quant(x, w, stream=stream)
        b = cake.cake_gemm_fp8(X, xs, W, wsc, stream=stream)
        c = cake.cake_kv_append(spare, k, v, slots, q=qs, stream=stream)
        d = cake.cake_paged_decode(q, cache, table, n, want_lse=True, stream=stream)
        return [a[0].view(torch.uint8), a[1], b, c, d[0], d[1]]

    want = run(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    sizes = [cake.cake_paged_decode_workspace_bytes(2, 32, 8, 128), cake.cake_gemm_fp8_workspace_bytes(100, 256, 4096), cake.CAKE_SERVING_HEADER_BYTES]
    for _ in range(3):
        dirty = [torch.full((m,), 85, dtype=torch.uint8, device=DEV) for m in sizes]      # what the current stream's allocator hands out next
        torch.cuda.synchronize()
        del dirty
        torch.cuda._sleep(20_000_000)                 # about 10 ms, in which nothing that is queued behind it runs
        got = run(side)
        scribble = [torch.full((m,), 85, dtype=torch.uint8, device=DEV) for m in sizes]
        side.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
        del scribble


@pytest.mark.parametrize("kv", [BF16, E4M3])
def test_keys_and_values_of_different_stride_orders(kv):
    """Keys token by token inside a page, values head by head (and rows further apart than they are long)."""
    g = gen(15)
    pages, page, Hkv, D = 12, 16, 4, 128
    k = torch.zeros(pages, page, Hkv, D + 16, device=DEV).to(kv)[..., :D]
    v = torch.zeros(pages, Hkv, page + 1, D, device=DEV).to(kv)[:, :, :page].transpose(1, 2)
    ks, vs = (torch.empty(Hkv, device=DEV).uniform_(0.01, 0.03, generator=g) if kv == E4M3 else None for _ in range(2))
    cache, plain = cake.PagedCache(k, v, ks, vs), cake.PagedCache(k.clone(memory_format=torch.contiguous_format), v.clone(memory_format=torch.contiguous_format), ks, vs)
    T = 150
    new_k, new_v = normal(g, T, Hkv, D), normal(g, T, Hkv, D)
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:T]
    for c in (cache, plain):
        cake.cake_kv_append(c, new_k, new_v, slots)
    for a, b in ((cache.k, plain.k), (cache.v, plain.v)):
        assert torch.equal(a.float(), b.float())
    q = normal(g, 3, 12, D)
    table = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).view(3, 4)
    n = torch.tensor([64, 1, 39], dtype=torch.int32, device=DEV)
    out, lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True)
    check_decode(q, cache, table, n, out, lse)
    assert torch.equal(out, cake.cake_paged_decode(q, plain, table, n)[0])


@pytest.mark.parametrize("B,Hq,Hkv,D,kv,start", [(16, 8, 2, 64, BF16, 40), (3, 16, 1, 128, E4M3, 9000), (150, 4, 4, 64, E4M3, 3),
                                                 (2, 4, 1, 128, BF16, 20000)])
def test_calls_back_to_back_give_the_bits_of_calls_one_by_one(B, Hq, Hkv, D, kv, start):
    """Every kernel may start before the one ahead of it ends: steps of a layer, each call writing what calls ahead of it still read, over the same few
    buffers; 60 steps with nothing between the launches, and as a graph, against the same steps with a wait after every call."""
    H, page, steps = 512, 16, 60
    g = gen(B)
    rows = (Hq + 2 * Hkv) * D
    w_in, w_out = normal(g, rows, H, std=1.0, dtype=E4M3), normal(g, H, Hq * D, std=1.0, dtype=E4M3)
    s_in = torch.full((-(-rows // 128), H // 128), 0.04, device=DEV)
    s_out = torch.full((H // 128, -(-Hq * D // 128)), 0.04, device=DEV)
    norm_w = normal(g, H, std=0.1) + 1
    width = -(-(start + steps) // page)
    table = torch.randperm(B * width, generator=g, device=DEV).to(torch.int32).view(B, width)
    at = start + torch.arange(steps, device=DEV)
    slots = (table[:, at // page].long() * page + at % page).t().contiguous()          # [steps, B]
    lens = (at + 1).to(torch.int32)[:, None].expand(steps, B).contiguous()
    pos, cos_sin = at.to(torch.int32)[:, None].expand(steps, B).contiguous(), rotary_table(start + steps, D)
    hidden = normal(g, B, H)
    old_k, old_v = (normal(g, B * width, page, Hkv, D, std=40.0 if kv == E4M3 else 1.0, dtype=kv) for _ in range(2))
    scale = torch.full((Hkv,), 0.02, device=DEV) if kv == E4M3 else None

    def run(wait, graph=False):
        cache = cake.PagedCache(old_k.clone(), old_v.clone(), scale, scale)
        x, res = hidden.clone(), torch.zeros_like(hidden)
        q8, sc = torch.empty(B, H, dtype=E4M3, device=DEV), torch.empty(B, H // 128, device=DEV)
        a8, asc = torch.empty(B, Hq * D, dtype=E4M3, device=DEV), torch.empty(B, -(-Hq * D // 128), device=DEV)
        proj = torch.empty(B, rows, dtype=BF16, device=DEV)
        heads = proj.view(B, Hq + 2 * Hkv, D)
        q, att = (torch.empty(B, Hq, D, dtype=BF16, device=DEV) for _ in range(2))
        ws, gws = cake.alloc_decode_workspace(B, Hq, Hkv, D, DEV), cake.alloc_gemm_workspace(None, rows, H, DEV)

        def step(t):
            for call in (lambda: cake.cake_rmsnorm_quant(x, norm_w, res, out_residual=res, out_q=q8, out_scale=sc),
                         lambda: cake.cake_gemm_fp8(q8, sc, w_in, s_in, out=proj, ws=gws),
                         lambda: cake.cake_kv_append(cache, heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:], slots[t], pos[t], cos_sin, q=heads[:, :Hq], out_q=q, ws=ws),
                         lambda: cake.cake_paged_decode(q, cache, table, lens[t], out=att, ws=ws),
                         lambda: cake.cake_rmsnorm_quant(att.view(B, -1), out_q=a8, out_scale=asc, flags=cake.CAKE_RMSNORM_NONE, want_residual=False),
                         lambda: cake.cake_gemm_fp8(a8, asc, w_out, s_out, out=x, ws=gws)):
                call()
                if wait:
                    torch.cuda.synchronize()

        if graph:
            torch.cuda.synchronize()
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                for t in range(steps):
                    step(t)
            captured.replay()
        else:
            for t in range(steps):
                step(t)
        torch.cuda.synchronize()
        assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK and cake.cake_kmeans_device_status(gws) == cake.CAKE_OK
        return [x, res, att, cache.k.view(torch.uint8), cache.v.view(torch.uint8)]

    want = run(True)
    assert torch.isfinite(want[0].float()).all() and (want[2] != 0).any()
    for got in (run(False), run(False), run(False, graph=True)):
        for a, b in zip(got, want):
            assert torch.equal(a, b)
