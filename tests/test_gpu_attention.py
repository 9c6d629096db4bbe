"""Attention of many query tokens (packed prompts, chunks over a paged cache) against a plain implementation in 64 bits.

Tolerances, from the arithmetic alone:
  weights  rounded to bf16 by at most half a step, 2^-8 (8-bit caches: f16, 2^-11, and 2^-32 of the heaviest, half a step of
           those that have no 11 bits, where the heaviest is at 2^7 or above):
           that share of sum p|v|
  scores   D products and sums in 32 bits, D 2^-23 sum|q k| scale, the scaling and 2^x another 8 of 2^-23 of the largest exponent: delta, which moves
           weights and their sum by as much
  sums     32 terms in each of four accumulators and one addition a tile of keys: (40 + n / 128) 2^-23
  out      then half a step of bf16, 2^-8 (1.01: the steps above it move it too)
"""
import math

import pytest
import torch

import paper_2608_12629_b200 as cake

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
U = 2.0 ** -23


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=BF16):
    return torch.empty(*shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def starts_of(lens):
    return torch.tensor([0] + list(lens), dtype=torch.int64).cumsum(0).to(torch.int32).to(DEV)


def visible(n, L, causal, window):
    p = L - n + torch.arange(n, device=DEV)[:, None]
    t = torch.arange(L, device=DEV)[None]
    if not causal:
        return torch.ones(n, L, dtype=torch.bool, device=DEV)
    ok = t <= p
    if window:
        ok &= t > p - window
    return ok


def reference(q, k, v, scale, seen):
    """q [n, G, D], k, v [L, D], seen [n, L] -> out, lse, and their bounds without the output's rounding, in 64 bits."""
    q, k, v = q.double(), k.double(), v.double()
    x = torch.einsum("igd,td->igt", q, k) * scale
    size = torch.einsum("igd,td->igt", q.abs(), k.abs()) * abs(scale)
    hide = ~seen[:, None, :].expand_as(x)
    x = x.masked_fill(hide, -math.inf)
    size = size.masked_fill(hide, 0.0)
    none = hide.all(2)
    lse = torch.logsumexp(x, 2)
    p = torch.exp(x - torch.where(none, torch.zeros_like(lse), lse)[..., None])
    vz = torch.where(seen.any(0)[:, None], v, torch.zeros_like(v))      # (values that no row sees)
    out = torch.einsum("igt,td->igd", p, vz)
    most = torch.einsum("igt,td->igd", p, vz.abs())
    n, D, L = q.shape[0], q.shape[2], k.shape[0]
    top = size.amax(2) if L else torch.zeros(n, q.shape[1], dtype=torch.float64, device=DEV)
    delta = D * U * top + 8 * U * (1.45 * top + 16)
    return out, lse, most, delta, none


def check(out, lse, q, keys_values, new, lens, Hkv, scale, causal, window, f16=False, keep=None, per_head=False):
    """keys_values(b, g) -> k, v [L, D] in fp32/64 as the attention sees them (scales applied); keep(b, g): keys that exist."""
    T, Hq, D = q.shape
    G = Hq // Hkv
    a, off, size = 0, 0.0, 0.0
    for b, n in enumerate(new):
        for g in range(Hkv):
            if n == 0:
                continue
            L = lens[b][g] if per_head else lens[b]
            k, v = keys_values(b, g)
            seen = visible(n, L, causal, window)
            if keep is not None:
                seen = seen & keep(b, g)[None, :]
            want, want_lse, most, delta, none = reference(q[a:a + n, g * G:(g + 1) * G], k, v, scale, seen)
            got, got_lse = out[a:a + n, g * G:(g + 1) * G].double(), lse[a:a + n, g * G:(g + 1) * G].double()
            sums = (40 + L / 128) * U
            bound = ((2.0 ** -11 if f16 else 2.0 ** -8) + 2 * delta + 2 * sums)[..., None] * most + 1.01 * 2.0 ** -8 * want.abs() + 1e-30
            if f16 and L:
                bound = bound + L * 2.0 ** -32 * v.double().abs().max()
            err = (got - want).abs()
            assert not (~(err <= bound)).any(), f"out of sequence {b}, head {g}: worst {float((err / bound).max()):.3g} bounds"
            assert (got[none] == 0).all() and (got_lse[none] == -math.inf).all()
            lerr = (got_lse - want_lse).abs()[~none]
            lbound = (delta + sums + 2.0 ** -22 + 2 * U * want_lse.abs())[~none]
            assert not (~(lerr <= lbound)).any(), f"lse of sequence {b}, head {g}: worst {float((lerr / lbound).max()):.3g} bounds"
            off, size = off + float(err.square().sum()), size + float(want.square().sum())
        a += n
    if out.numel() > 4096:
        # roundings of weights and output, each uniform in half a step at most: 2^-8 / sqrt(3) apart, independent
        assert off <= (2.0 / 3) * 2.0 ** -16 * size, f"error of {math.sqrt(off / size):.4g} in norm"


def packed(seed, new, lens, Hq, Hkv, D, std=1.2, extra=0):
    g = gen(seed)
    T, Tk = sum(new) + extra, sum(lens) + extra
    q, k, v = normal(g, T, Hq, D, std=std), normal(g, Tk, Hkv, D, std=std), normal(g, Tk, Hkv, D)
    return q, k, v


def run_packed(q, k, v, new, lens, causal=True, window=0, scale=None, **more):
    ws = cake.alloc_attention_workspace(q.shape[1], k.shape[1], q.shape[2], DEV)
    out, lse = cake.cake_prompt_attention(q, k, v, starts_of(new), None if new is lens else starts_of(lens), causal=causal, window=window, scale=scale,
                                          want_lse=True, ws=ws, **more)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK
    return out, lse


def check_packed(out, lse, q, k, v, new, lens, causal=True, window=0, scale=None):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    check(out, lse, q, lambda b, g: (k[at[b]:at[b + 1], g], v[at[b]:at[b + 1], g]), new, lens, k.shape[1],
          q.shape[2] ** -0.5 if scale is None else scale, causal, window)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (6, 2), (8, 8)])
@pytest.mark.parametrize("lens", [[1], [5], [128], [129], [127, 0, 1, 300], [700, 31]])
def test_prompt_shapes(D, Hq, Hkv, lens):
    q, k, v = packed(sum(lens) + D + Hq, lens, lens, Hq, Hkv, D)
    for causal in (True, False):
        out, lse = run_packed(q, k, v, lens, lens, causal)
        check_packed(out, lse, q, k, v, lens, lens, causal)


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 5, 1), (64, 16, 1), (96, 7, 7), (128, 32, 8), (128, 65, 1), (128, 3, 1), (128, 130, 1), (128, 300, 2), (256, 12, 4)])
def test_prompt_groups_of_any_size(D, Hq, Hkv):
    """Groups that do not divide a tile of 128 rows, that fill it, and that pass it."""
    lens = [150, 40, 1]
    q, k, v = packed(Hq, lens, lens, Hq, Hkv, D)
    out, lse = run_packed(q, k, v, lens, lens)
    check_packed(out, lse, q, k, v, lens, lens)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("window", [1, 7, 128, 200, 4000])
def test_prompt_windows(D, window):
    lens = [900, 1, 260]
    q, k, v = packed(window, lens, lens, 4, 2, D)
    out, lse = run_packed(q, k, v, lens, lens, window=window)
    check_packed(out, lse, q, k, v, lens, lens, window=window)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_keys_of_another_length(D, causal):
    """Behind a prefix, without keys, and with fewer keys than tokens: the first tokens then see nothing."""
    new, lens = [5, 130, 3, 300, 64], [517, 130, 0, 100, 1000]
    q, k, v = packed(D, new, lens, 4, 2, D)
    for window in (0, 90) if causal else (0,):
        out, lse = run_packed(q, k, v, new, lens, causal, window)
        check_packed(out, lse, q, k, v, new, lens, causal, window)


@pytest.mark.parametrize("D,Hq,Hkv,lens", [(128, 8, 2, [5000, 333]), (64, 4, 4, [6000]), (256, 4, 1, [3001]), (96, 6, 2, [2500, 2500]), (128, 2, 1, [9000]),
                                           (128, 16, 8, [200] * 50)])
def test_prompt_long_and_split(D, Hq, Hkv, lens):
    """Items that several CTAs share, rescaled sums over many tiles, more items than CTAs; the same bits every time from the same workspace."""
    q, k, v = packed(D + Hq, lens, lens, Hq, Hkv, D)
    q[1::7] *= 6.0                                  # rows whose maximum keeps moving
    out, lse = run_packed(q, k, v, lens, lens)
    check_packed(out, lse, q, k, v, lens, lens)
    ws = cake.alloc_attention_workspace(Hq, Hkv, D, DEV)
    s = starts_of(lens)
    for _ in range(3):
        again, lse2 = cake.cake_prompt_attention(q, k, v, s, want_lse=True, ws=ws)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_prompt_scales(scale):
    lens = [200, 129]
    q, k, v = packed(1, lens, lens, 4, 2, 64)
    out, lse = run_packed(q, k, v, lens, lens, scale=scale)
    check_packed(out, lse, q, k, v, lens, lens, scale=scale)


def test_prompt_strides_and_rows_behind_the_last_sequence():
    """Views of one projection, heads outermost, and tokens of no sequence, which stay as they were."""
    g = gen(8)
    lens, Hq, Hkv, D = [100, 0, 77], 6, 2, 128
    T = sum(lens)
    rows = normal(g, T + 9, Hq + 2 * Hkv, D)
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    out = torch.full((T + 9, Hq, D), 7.0, dtype=BF16, device=DEV)
    lse = torch.full((T + 9, Hq), 5.0, device=DEV)
    cake.cake_prompt_attention(q, k, v, starts_of(lens), out=out, out_lse=lse)
    check_packed(out, lse, q, k, v, lens, lens)
    assert (out[T:] == 7).all() and (lse[T:] == 5).all()
    # sequences that begin behind the first token leave those before it
    out2 = torch.full_like(out, 7.0)
    cake.cake_prompt_attention(q, k, v, starts_of(lens)[1:], out=out2)
    assert (out2[:100] == 7).all() and torch.equal(out2[100:T], out[100:T]) and (out2[T:] == 7).all()
    heads_first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    out3, _ = cake.cake_prompt_attention(*heads_first, starts_of(lens), out=torch.full_like(out, 7.0))
    assert torch.equal(out3, out)


def test_prompt_values_that_are_not_finite():
    """Infinities and NaN of tokens that a row does not see leave it alone; of those that it sees they reach it."""
    lens, Hq, Hkv, D = [300, 260], 4, 2, 128
    q, k, v = packed(3, lens, lens, Hq, Hkv, D)
    clean, clean_lse = run_packed(q, k, v, lens, lens)
    for bad in (math.nan, math.inf):
        k2, v2 = k.clone(), v.clone()
        v2[200, 0, 5] = bad                         # a value of the first sequence's token 200, head 0
        k2[450, 1, 9] = math.nan                    # a key of the second's token 150, head 1
        v2[300:310] = bad                           # the second's first ten values: none of the first sequence's
        out, lse = run_packed(q, k2, v2, lens, lens)
        assert torch.equal(out[:200], clean[:200]) or float((out[:200].float() - clean[:200].float()).abs().max()) < 0.02
        assert torch.isfinite(out[:300, 2:]).all() and torch.isfinite(lse[:300]).all()
        hit = out[200:300, :2]
        assert not torch.isfinite(hit[..., 5]).any() and torch.isfinite(hit[..., :5]).all() and torch.isfinite(hit[..., 6:]).all()
        assert torch.isnan(lse[450:, 2:]).all() and torch.isfinite(lse[300:450]).all() and torch.isfinite(lse[:, :2]).all()
        assert not torch.isfinite(out[300:]).any()
    # a whole sequence of them beside another
    k2, v2 = k.clone(), v.clone()
    k2[300:], v2[300:] = math.nan, math.nan
    out, lse = run_packed(q, k2, v2, lens, lens)
    check_packed(out[:300], lse[:300], q[:300], k2[:300], v2[:300], lens[:1], lens[:1])
    assert torch.isnan(out[300:]).all()
    # windows: what lies before them
    v2 = v.clone()
    v2[:50] = math.nan
    out, lse = run_packed(q, k, v2, lens, lens, window=40)
    ref, _ = run_packed(q, k, v, lens, lens, window=40)
    assert float((out[89:].float() - ref[89:].float()).abs().max()) < 0.02 and torch.isnan(out[:89]).all()


def test_prompt_rows_that_see_nothing_beside_values_that_are_not_finite():
    q, k, v = packed(4, [300], [100], 2, 1, 64)
    v[:] = math.nan
    out, lse = run_packed(q, k, v, [300], [100])
    assert (out[:200] == 0).all() and (lse[:200] == -math.inf).all() and torch.isnan(out[200:]).all()


def test_prompt_infinite_scores():
    """A key whose products are -inf weighs nothing; rows of which all are -inf are NaN or nothing, as the softmax says, and leave the others alone."""
    q, k, v = packed(5, [64], [64], 2, 1, 64)
    q[:] = q.abs().clamp(min=0.1)
    k[7] = -math.inf
    out, lse = run_packed(q, k, v, [64], [64])
    keep = torch.ones(64, dtype=torch.bool, device=DEV)
    keep[7] = False
    k2 = k.clone()
    k2[7] = 0
    check(out, lse, q, lambda b, g: (k2[:, g], v[:, g]), [64], [64], 1, 64 ** -0.5, True, 0, keep=lambda b, g: keep)


# ------------------------------------------------------------------------------------------------------------ chunks
def paged(seed, new, lens, Hq, Hkv, D, page, kv, std=1.2, spare=2, by_head=False):
    g = gen(seed)
    need = [max(-(-n // page), 0) for n in lens]
    pages, width = sum(need) + spare, max(max(need), 1)
    order = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (pages, Hkv, page, D) if by_head else (pages, page, Hkv, D)
    scales = (None, None)
    if kv == "e4m3":
        kc, vc = (normal(g, *shape, std=60.0, dtype=E4M3) for _ in range(2))
        scales = tuple(torch.empty(Hkv, device=DEV).uniform_(0.01, 0.025, generator=g) for _ in range(2))
    else:
        kc, vc = (normal(g, *shape) for _ in range(2))
    # what no sequence holds is not finite
    used = torch.zeros(pages, page, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        t = torch.arange(n, device=DEV)
        used[table[b, t // page].long(), t % page] = True
    for c in (kc, vc):
        bits = c.view(torch.uint8 if kv == "e4m3" else torch.int16)
        bits = bits.transpose(1, 2) if by_head else bits
        bits[~used] = 0x7f if kv == "e4m3" else 0x7fc0
    if by_head:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    q = normal(g, sum(new), Hq, D, std=std)
    return q, cake.PagedCache(kc, vc, *scales), table, torch.tensor(lens, dtype=torch.int32, device=DEV)


def cached(cache, table, lens, b, g):
    t = torch.arange(lens[b], device=DEV)
    where = (table[b, t // cache.page_size].long().clamp(min=0), t % cache.page_size)
    k, v = (x[:, :, g][where].double() for x in (cache.k, cache.v))
    if cache.k_scale is not None:
        k, v = k * cache.k_scale[g].double(), v * cache.v_scale[g].double()
    return k, v


def run_chunk(q, cache, table, lens, new, window=0, scale=None):
    ws = cake.alloc_attention_workspace(q.shape[1], cache.Hkv, cache.D, DEV)
    out, lse = cake.cake_paged_chunk(q, cache, table, lens, starts_of(new), window=window, scale=scale, want_lse=True, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK
    return out, lse


def check_chunk(out, lse, q, cache, table, new, lens, window=0, scale=None, keep=None):
    check(out, lse, q, lambda b, g: cached(cache, table, lens, b, g), new, lens, cache.Hkv, cache.D ** -0.5 if scale is None else scale, True, window,
          f16=cache.k.dtype == E4M3, keep=keep)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("page,new,lens", [
    (16, [1], [1]), (16, [1], [500]), (1, [3], [130]), (100, [7, 1, 0, 40], [301, 1, 5, 40]), (64, [200, 1], [200, 900]), (128, [129], [1000]),
    (8, [300, 33], [300, 700]), (300, [2], [257])])
def test_chunk_shapes(kv, D, page, new, lens):
    q, cache, table, n = paged(page + sum(lens), new, lens, 4, 2, D, page, kv, by_head=page == 64)
    out, lse = run_chunk(q, cache, table, n, new)
    check_chunk(out, lse, q, cache, table, new, lens)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 3, 1), (96, 12, 1), (128, 20, 4), (128, 64, 8), (128, 140, 1), (256, 6, 2)])
def test_chunk_groups_of_any_size(kv, D, Hq, Hkv):
    new, lens = [4, 1, 150], [333, 64, 700]
    q, cache, table, n = paged(Hq, new, lens, Hq, Hkv, D, 16, kv)
    for window in (0, 100):
        out, lse = run_chunk(q, cache, table, n, new, window)
        check_chunk(out, lse, q, cache, table, new, lens, window)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq,Hkv,new,lens", [(128, 8, 1, [4], [30001]), (64, 8, 4, [1] * 40, [50 * i + 1 for i in range(40)]), (256, 4, 1, [9, 1], [7000, 20]),
                                               (128, 16, 4, [1000, 1, 1, 1], [9000, 1, 5000, 300]), (96, 4, 4, [2, 600], [12000, 600])])
def test_chunk_long_and_split(kv, D, Hq, Hkv, new, lens):
    q, cache, table, n = paged(D + Hq, new, lens, Hq, Hkv, D, 64, kv)
    out, lse = run_chunk(q, cache, table, n, new)
    check_chunk(out, lse, q, cache, table, new, lens)
    for _ in range(3):
        again, lse2 = run_chunk(q, cache, table, n, new)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_chunk_pages_out_of_range_are_left_out(kv):
    """Their keys weigh nothing, and the status says so; entries that no token sees are not looked at."""
    page, new, lens = 16, [20, 3], [500, 90]
    q, cache, table, n = paged(2, new, lens, 4, 2, 128, page, kv)
    keep = torch.ones(2, 500, dtype=torch.bool, device=DEV)
    for b, entry, value in ((0, 3, -7), (0, 20, cache.num_pages), (1, 0, -2 ** 31)):
        table[b, entry] = value
        keep[b, entry * page:(entry + 1) * page] = False
    ws = cake.alloc_attention_workspace(4, 2, 128, DEV)
    out, lse = cake.cake_paged_chunk(q, cache, table, n, starts_of(new), want_lse=True, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    held = table.clone()
    table[:] = held.clamp(0, cache.num_pages - 1)
    check(out, lse, q, lambda b, g: tuple(torch.nan_to_num(x) for x in cached(cache, table, lens, b, g)), new, lens, 2, 128 ** -0.5, True, 0, f16=kv == "e4m3",
          keep=lambda b, g: keep[b, :lens[b]])
    table[:] = held
    table[0, :20] = 10 ** 6                          # before the window, and behind the sequence
    table[1, 6:] = 10 ** 6
    table[0, 20] = table[0, 21]
    table[1, 0] = table[1, 1]
    ws = cake.alloc_attention_workspace(4, 2, 128, DEV)
    out, lse = cake.cake_paged_chunk(q, cache, table, n, starts_of(new), want_lse=True, ws=ws, window=100)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK
    check_chunk(out, lse, q, cache, table.clamp(0, cache.num_pages - 1), new, lens, 100)


def test_chunk_lengths_out_of_range():
    q, cache, table, n = paged(2, [5, 5], [40, 40], 4, 2, 64, 16, "bf16")
    ws = cake.alloc_attention_workspace(4, 2, 64, DEV)
    n[0], n[1] = 1000, -3                            # cut to the table's 48 tokens; none
    out, lse = cake.cake_paged_chunk(q, cache, table, n, starts_of([5, 5]), want_lse=True, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    assert (out[5:] == 0).all() and (lse[5:] == -math.inf).all()
    for starts in ([0, 11, 10], [-1, 5, 10], [6, 5, 10]):      # the first sequence is left out
        out = torch.full_like(q, 3.0)
        ws = cake.alloc_attention_workspace(4, 2, 64, DEV)
        n[0], n[1] = 40, 40
        cake.cake_paged_chunk(q, cache, table, n, torch.tensor(starts, dtype=torch.int32, device=DEV), out=out, ws=ws)
        assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
        if starts != [0, 11, 10]:
            assert (out[:5] == 3).all() and (out[5:] != 3).any()
        else:
            assert (out == 3).all()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_chunk_of_one_token_is_a_decode(kv):
    """Against the decode of the same tokens, with a table and a length per head too."""
    new, lens = [1] * 5, [700, 1, 64, 129, 2000]
    q, cache, table, n = paged(9, new, lens, 8, 2, 128, 16, kv)
    out, lse = run_chunk(q, cache, table, n, new)
    ref, ref_lse = cake.cake_paged_decode(q, cache, table, n, want_lse=True)
    assert float((out.float() - ref.float()).abs().max()) < 0.02 and float((lse - ref_lse).abs().max()) < 1e-4
    per = table[:, None].repeat(1, 2, 1)
    per[0, 1] = per[0, 1].flip(0)
    ln = torch.stack([n, (n + 1) // 2], 1).contiguous()
    per[0, 1, :22] = table[0, :22]
    ws = cake.alloc_attention_workspace(8, 2, 128, DEV)
    out, lse = cake.cake_paged_chunk(q, cache, per, ln, starts_of(new), want_lse=True, ws=ws)
    ref, ref_lse = cake.cake_paged_decode(q, cache, per, ln, want_lse=True)
    assert float((out.float() - ref.float()).abs().max()) < 0.02 and float((lse - ref_lse).abs().max()) < 1e-4


def test_chunk_of_a_whole_prompt_is_the_prompt():
    new = [300, 77, 1]
    q, cache, table, n = paged(11, new, new, 4, 2, 128, 32, "bf16")
    out, lse = run_chunk(q, cache, table, n, new)
    k, v = (torch.cat([torch.stack([cached(cache, table, new, b, g)[i] for g in range(2)], 1) for b in range(3)]).to(BF16) for i in range(2))
    ref, ref_lse = run_packed(q, k, v, new, new)
    # (the same tiles in the same order: the same bits)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)


def test_chunk_tiny_and_huge_queries_over_an_8_bit_cache():
    """Queries are brought to 16 bits by powers of two, a row at a time."""
    new, lens = [6], [300]
    q, cache, table, n = paged(12, new, lens, 4, 2, 128, 16, "e4m3")
    q[0], q[1], q[2], q[3, 0] = q[0] * 2.0 ** -100, q[1] * 2.0 ** 5, 0.0, 0.0
    out, lse = run_chunk(q, cache, table, n, new)
    check_chunk(out, lse, q, cache, table, new, lens)


def test_no_tokens_and_refusals():
    q, k, v = packed(1, [4], [4], 4, 2, 64)
    s = starts_of([4])
    assert cake.cake_prompt_attention(q[:0], k[:0], v[:0], starts_of([0]))[0].shape == (0, 4, 64)
    assert cake.cake_prompt_attention(q, k, v, starts_of([]), out=torch.full_like(q, 3.0))[0].eq(3).all()
    out, lse = cake.cake_prompt_attention(q, k[:0], v[:0], s, starts_of([0]), want_lse=True)      # no keys at all
    assert (out == 0).all() and (lse == -math.inf).all()
    for args, code in (((q[..., :32], k[..., :32], v[..., :32]), cake.CAKE_ERR_UNSUPPORTED), ((q[:, :3], k, v), cake.CAKE_ERR_SHAPE)):
        with pytest.raises(cake.CakeError) as e:
            cake.cake_prompt_attention(*args, s, ws=cake.alloc_attention_workspace(4, 2, 64, DEV))
        assert e.value.code == code
    with pytest.raises(cake.CakeError) as e:
        cake.cake_prompt_attention(q, k, v, s, causal=False, window=3)
    assert e.value.code == cake.CAKE_ERR_UNSUPPORTED
    with pytest.raises(cake.CakeError) as e:
        cake.cake_prompt_attention(q, k, v, s, ws=torch.zeros(20000, dtype=torch.uint8, device=DEV))
    assert e.value.code == cake.CAKE_ERR_WORKSPACE
    odd = normal(gen(1), 4, 4 * 64 + 4)[:, 4:].view(4, 4, 64)
    for args in ((odd, k, v), (q, odd[:, :2], v)):
        with pytest.raises(cake.CakeError) as e:
            cake.cake_prompt_attention(*args, s)
        assert e.value.code == cake.CAKE_ERR_ALIGN
    with pytest.raises(cake.CakeError) as e:
        cake.cake_prompt_attention(q, k[:1].expand(4, 2, 64), v, s)
    assert e.value.code == cake.CAKE_ERR_SHAPE
    for bad in (dict(starts=s.long()), dict(starts=s[None]), dict(k=k.float()), dict(out=torch.zeros(4, 4, 32, dtype=BF16, device=DEV)),
                dict(out_lse=torch.zeros(4, 4, dtype=BF16, device=DEV)), dict(ws=torch.zeros(64, device=DEV))):
        with pytest.raises(TypeError):
            cake.cake_prompt_attention(**{**dict(q=q, k=k, v=v, starts=s), **bad})
    with pytest.raises(ValueError):
        cake.cake_prompt_attention(q, k, v[:3], s)
    with pytest.raises(ValueError):
        cake.cake_prompt_attention(q, k, v, s, starts_of([2, 2]))
    qc, cache, table, n = paged(1, [2], [20], 4, 2, 64, 16, "bf16")
    for bad in (dict(starts=starts_of([1, 1])), dict(seq_lens=n.repeat(2)), dict(page_table=table.repeat(2, 1))):
        with pytest.raises(ValueError):
            cake.cake_paged_chunk(**{**dict(q=qc, cache=cache, page_table=table, seq_lens=n, starts=starts_of([2])), **bad})
    for bad in (dict(page_table=table.long()), dict(q=qc.float())):
        with pytest.raises(TypeError):
            cake.cake_paged_chunk(**{**dict(q=qc, cache=cache, page_table=table, seq_lens=n, starts=starts_of([2])), **bad})


@pytest.mark.parametrize("D,kv", [(64, "bf16"), (128, "bf16"), (256, "bf16"), (128, "e4m3"), (256, "e4m3")])
@pytest.mark.parametrize("up", [True, False])
def test_scores_that_grow_or_fall_along_the_sequence(D, kv, up):
    """A maximum that rises by hundreds from tile to tile is followed (what went before then weighs nothing); one that falls is kept."""
    new, lens = [70, 3], [1500, 900]
    q, cache, table, n = paged(21, new, lens, 4, 2, D, 16, kv)
    q.abs_().clamp_(min=0.05)
    g = gen(22)
    for b, L in enumerate(lens):
        t = torch.arange(L, device=DEV)
        where = (table[b, t // 16].long(), t % 16)
        size = (t if up else L - t).float() / L * (400 if kv == "e4m3" else 40)
        rows = size[:, None, None] * (0.9 + 0.1 * torch.rand(L, 2, D, generator=g, device=DEV))
        if kv == "e4m3":
            cache.k.view(torch.uint8)[where] = rows.to(E4M3).view(torch.uint8)
        else:
            cache.k[where] = rows.to(BF16)
    out, lse = run_chunk(q, cache, table, n, new)
    check_chunk(out, lse, q, cache, table, new, lens)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_huge_scores_do_not_hang_and_follow_the_largest():
    """Scores of 10^30 and more, whose differences 32 bits do not hold: the calls end, and rows with one largest key give its value."""
    lens = [260]
    q, k, v = packed(23, lens, lens, 2, 1, 64)
    q[:] = 2.0 ** 60
    k[:] = 0
    k[7, 0, 0] = 2.0 ** 60
    out, lse = run_packed(q, k, v, lens, lens)
    assert torch.equal(out[7:], v[7].expand(253, 2, 64)) and torch.isfinite(out[:7]).all()
    k[:] = torch.randn(260, 1, 64, device=DEV).bfloat16() * 2.0 ** 60
    out, lse = run_packed(q, k, v, lens, lens)
    assert out.shape == q.shape
