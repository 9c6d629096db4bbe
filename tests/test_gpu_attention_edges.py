"""Attention of many tokens at the edges of its range, against a plain implementation in 64 bits: scales that are no numbers or next to nothing, scores and values
beyond what 32 bits add up, values that are not finite and not seen, ranges out of bounds, the lightest weights of 8-bit caches, pieces of prompts as they are used.

Tolerances: those of test_gpu_attention.py, whose reference and bounds this file uses."""
import math

import pytest
import torch

import paper_2608_12629_b200 as cake
from tests import test_gpu_attention as base

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def nothing(n, L):
    """Tokens of n that see none of L keys."""
    return max(n - L, 0)


# -------------------------------------------------------------------------------------------------------------- scales
@pytest.mark.parametrize("D,lens", [(64, [70, 300]), (128, [3000]), (256, [5, 1500])])
def test_a_scale_that_is_no_number_reaches_every_row_that_sees_something(D, lens):
    """Whole items and items that several CTAs share; tokens that see nothing stay zeros."""
    keys = [n - 3 for n in lens]
    q, k, v = base.packed(D, lens, keys, 4, 2, D)
    out, lse = base.run_packed(q, k, v, lens, keys, scale=math.nan)
    at = 0
    for n, L in zip(lens, keys):
        none = nothing(n, L)
        assert (out[at:at + none] == 0).all() and (lse[at:at + none] == -math.inf).all()
        assert torch.isnan(out[at + none:at + n]).all() and torch.isnan(lse[at + none:at + n]).all()
        at += n


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,lens", [([3, 200], [40, 500]), ([5], [4000])])
def test_a_scale_that_is_no_number_over_pages(kv, new, lens):
    q, cache, table, n = base.paged(4, new, lens, 4, 2, 128, 16, kv)
    out, lse = base.run_chunk(q, cache, table, n, new, scale=math.nan)
    assert torch.isnan(out).all() and torch.isnan(lse).all()
    if kv == "e4m3":                                  # of one head alone
        cache.k_scale[1] = math.nan
        out, lse = base.run_chunk(q, cache, table, n, new)
        assert torch.isnan(out[:, 2:]).all() and torch.isnan(lse[:, 2:]).all()
        cache.k_scale[1] = 0.02
        want, want_lse = base.run_chunk(q, cache, table, n, new)
        assert torch.equal(out[:, :2], want[:, :2]) and torch.equal(lse[:, :2], want_lse[:, :2])


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("sign", [1, -1])
def test_scales_next_to_nothing_of_products_next_to_infinity(D, sign):
    """Scores of ordinary size from queries and keys of 2^60 and a scale of 2^-120; and products of 2^110 under a scale of zero, which weigh alike."""
    lens = [300, 33]
    q, k, v = base.packed(D, lens, lens, 4, 2, D)
    q, k = q * 2.0 ** 60, k * 2.0 ** 60
    scale = sign * 2.0 ** -120 * D ** -0.5
    out, lse = base.run_packed(q, k, v, lens, lens, scale=scale)
    base.check_packed(out, lse, q, k, v, lens, lens, scale=scale)
    q, k = q * 2.0 ** -5, k * 2.0 ** -5
    out, lse = base.run_packed(q, k, v, lens, lens, scale=0.0)
    base.check_packed(out, lse, q, k, v, lens, lens, scale=0.0)


def test_scales_of_an_8_bit_cache_whose_product_leaves_32_bits_on_the_way():
    """scale 2^-69 and a keys' scale of about 2^-66 make 2^-135; queries of 2^125 bring the scores back."""
    new, lens = [3, 140], [50, 300]
    q, cache, table, n = base.paged(11, new, lens, 4, 2, 128, 16, "e4m3")
    cache.k_scale.mul_(2.0 ** -60)
    q *= 2.0 ** 125
    assert torch.isfinite(q).all()
    out, lse = base.run_chunk(q, cache, table, n, new, scale=2.0 ** -69)
    base.check_chunk(out, lse, q, cache, table, new, lens, scale=2.0 ** -69)


# -------------------------------------------------------------------------------------------------------- large scores
def check_largest(out, lse, q, keys_values, new, lens, Hkv, scale, top):
    """Scores so far apart that all but a row's largest weigh nothing.  Where the largest leads the next by more than their roundings, (D + 3) 2^-23 of sum |q k|, and
    another 200 for the weights, the row is its value (its weight and the output rounded), and lse its score; where not, it lies between the values and the lse within
    that much of it."""
    T, Hq, D = q.shape
    G, at, clear = Hq // Hkv, 0, 0
    for b, n in enumerate(new):
        for g in range(Hkv):
            k, v = (t.double() for t in keys_values(b, g))
            rows = q[at:at + n, g * G:(g + 1) * G].double()
            hide = ~base.visible(n, lens[b], True, 0)[:, None, :].expand(n, G, lens[b])
            x = (torch.einsum("igd,td->igt", rows, k) * scale).masked_fill(hide, -math.inf)
            err = (D + 3) * base.U * (torch.einsum("igd,td->igt", rows.abs(), k.abs()) * abs(scale)).masked_fill(hide, 0).amax(2)
            assert float(x.amax()) > top
            best, where = x.max(2)
            next_best = x.scatter(2, where[..., None], -math.inf).amax(2)
            lead = best - next_best > 2 * err + 200
            got, got_lse = out[at:at + n, g * G:(g + 1) * G].double(), lse[at:at + n, g * G:(g + 1) * G].double()
            assert ((got - v[where]).abs() <= 2.01 * 2.0 ** -8 * v[where].abs())[lead].all()
            assert (got.abs() <= 1.01 * v.abs().max()).all()
            assert ((got_lse - best).abs() <= err + 2 * base.U * best.abs() + 10).all()
            clear += int(lead.sum())
        at += n
    assert clear > T * Hq // 2


@pytest.mark.parametrize("power", [11, 13, 30, 58])
@pytest.mark.parametrize("D,lens", [(64, [260, 5]), (96, [130]), (128, [2500]), (256, [1300, 40])])
def test_scores_far_beyond_what_their_differences_leave_in_32_bits(D, lens, power):
    """Scores of 2^23 to 2^118: their maximum's rounding alone would pass the range of an exponential."""
    q, k, v = base.packed(D, lens, lens, 4, 2, D)
    q, k = q * 2.0 ** power, k * 2.0 ** power
    out, lse = base.run_packed(q, k, v, lens, lens)
    at = [0, lens[0], sum(lens)]
    check_largest(out, lse, q, lambda b, g: (k[at[b]:at[b + 1], g], v[at[b]:at[b + 1], g]), lens, lens, 2, D ** -0.5, 2.0 ** (2 * power))
    # most of a row's keys and then the others as they are: its scores come into the range again, the other way round they leave it
    for part in (slice(0, sum(lens) // 2), slice(sum(lens) // 2, None)):
        k2 = k.clone()
        k2[part] = k2[part] * 2.0 ** -power
        out, lse = base.run_packed(q, k2, v, lens, lens)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all() and (out.abs() <= 1.01 * v.abs().max()).all()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,new,lens", [(128, [200, 3], [300, 4000]), (256, [9], [1500])])
def test_scores_beyond_over_pages(kv, D, new, lens):
    q, cache, table, n = base.paged(5, new, lens, 4, 2, D, 16, kv)
    q *= 2.0 ** 60
    out, lse = base.run_chunk(q, cache, table, n, new)
    check_largest(out, lse, q, lambda b, g: base.cached(cache, table, lens, b, g), new, lens, 2, D ** -0.5, 2.0 ** 60)


def test_ordinary_rows_beside_rows_of_large_scores():
    """A row's bits do not depend on its neighbours, whose scores take another way."""
    lens = [300, 2000]
    q, k, v = base.packed(6, lens, lens, 4, 2, 128)
    want, want_lse = base.run_packed(q, k, v, lens, lens)
    q2 = q.clone()
    q2[::3] *= 2.0 ** 80
    q2[1::6, 1] *= -2.0 ** 40
    out, lse = base.run_packed(q2, k, v, lens, lens)
    same = (q2 == q).all(2)
    assert torch.equal(out[same], want[same]) and torch.equal(lse[same], want_lse[same]) and torch.isfinite(out).all() and torch.isfinite(lse).all()


# ------------------------------------------------------------------------------------------------------------- ranges
@pytest.mark.parametrize("k_starts", [[0, 50, 40, 90], [0, 50, -1, 90], [0, 50, 100, 90], None])
def test_sequences_whose_keys_are_out_of_range_are_left_out(k_starts):
    """Their tokens stay as they were; the others' are theirs.  k_starts None: 90 keys for 120 tokens, which the last sequence's pass."""
    g = base.gen(3)
    new, D = [40, 30, 50], 64
    q, k, v = base.normal(g, 120, 4, D, std=1.2), base.normal(g, 90, 2, D, std=1.2), base.normal(g, 90, 2, D)
    ks = None if k_starts is None else torch.tensor(k_starts, dtype=torch.int32, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((120, 4), 5.0, device=DEV)
    ws = cake.alloc_attention_workspace(4, 2, D, DEV)
    cake.cake_prompt_attention(q, k, v, base.starts_of(new), ks, out=out, out_lse=lse, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    at = k_starts or [0, 40, 70, 120]
    a = 0
    for b, n in enumerate(new):
        k0, k1 = at[b], at[b + 1]
        if 0 <= k0 <= k1 <= 90:
            base.check_packed(out[a:a + n], lse[a:a + n], q[a:a + n], k[k0:k1], v[k0:k1], [n], [k1 - k0])
        else:
            assert (out[a:a + n] == 7).all() and (lse[a:a + n] == 5).all()
        a += n


def test_lengths_beyond_the_table_and_sequences_beside_those_that_are_left_out():
    """A length beyond the table is cut to it: 48 tokens; sequences beside one whose starts are out of range are theirs."""
    q, cache, table, n = base.paged(2, [5, 5], [48, 40], 4, 2, 64, 16, "bf16")
    ws = cake.alloc_attention_workspace(4, 2, 64, DEV)
    n[0] = 1000
    out, lse = cake.cake_paged_chunk(q, cache, table, n, base.starts_of([5, 5]), want_lse=True, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    base.check_chunk(out, lse, q, cache, table, [5, 5], [48, 40])
    for starts, kept in (([-1, 5, 10], 1), ([6, 5, 10], 1), ([0, 5, 4], 0), ([0, 5, 11], 0)):
        out, lse = torch.full_like(q, 3.0), torch.full((10, 4), 2.0, device=DEV)
        n[0] = 48
        cake.cake_paged_chunk(q, cache, table, n, torch.tensor(starts, dtype=torch.int32, device=DEV), out=out, out_lse=lse, ws=ws)
        mine, other = slice(5 * kept, 5 * kept + 5), slice(5 - 5 * kept, 10 - 5 * kept)
        assert (out[other] == 3).all() and (lse[other] == 2).all()
        base.check_chunk(out[mine], lse[mine], q[mine], cache, table[kept:kept + 1], [5], [[48, 40][kept]])


# ------------------------------------------------------------------------- values that are not finite, seen and not seen
def check_around(out, lse, q, keys_values, new, lens, Hkv, bad, window=0, keep=None, **more):
    """bad: {(sequence, token): columns} whose values are not finite.  Tokens that see none of them are theirs; of the others the columns named are not finite, the rest theirs."""
    scale, a = q.shape[2] ** -0.5, 0
    for b, n in enumerate(new):
        marks = sorted(t for s, t in bad if s == b)
        cuts = sorted({0, *(min(max(t - (lens[b] - n), 0), n) for t in marks), *(min(max(t - (lens[b] - n) + window, 0), n) for t in marks if window), n})
        for i0, i1 in zip(cuts[:-1], cuts[1:]):
            L = lens[b] - n + i1                      # these tokens' keys
            first = max(0, L - (i1 - i0) - window + 1) if window else 0      # of the first of them
            seen = [t for t in marks if t < L and t >= (L - window if window else 0)]
            cols = sorted({c for t in seen for c in bad[b, t]})
            sub, sub_lse = out[a + i0:a + i1].clone(), lse[a + i0:a + i1]
            assert not torch.isfinite(sub[..., cols]).any()
            sub[..., cols] = 0

            def without(_, g):
                k, v = (t[:L].double().clone() for t in keys_values(b, g))
                for t in marks:
                    if t < L:
                        v[t, list(bad[b, t])] = 0
                v[:, cols] = 0
                return k, v
            base.check(sub, sub_lse, q[a + i0:a + i1], without, [i1 - i0], [L], Hkv, scale, True, window,
                       keep=None if keep is None else lambda _, g: keep[b, :L], **more)
        a += n


NOT_FINITE = [(D, new, lens, window) for D in (64, 96, 128, 256) for new, lens, window in
              (([200, 5], [330, 130], 0), ([3], [4001], 0), ([70, 300], [2500, 300], 0), ([150, 260], [1700, 900], 77))]


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,new,lens,window", NOT_FINITE)
def test_chunk_values_that_are_not_finite(kv, D, new, lens, window):
    """Whole items and parts of them, two row tiles and one, pages that are missing."""
    page = 16
    q, cache, table, n = base.paged(D + window, new, lens, 4, 2, D, page, kv)
    g = base.gen(D)
    bad, keep = {}, torch.ones(len(new), max(lens), dtype=torch.bool, device=DEV)
    missing = [(b, max(L - m, 0) // 2 // page) for b, (m, L) in enumerate(zip(new, lens)) if L > m + 2 * page]
    for b, (m, L) in enumerate(zip(new, lens)):
        for t, cols in ((L - 1, range(D)), (L - 1 - m // 3, (3, D - 1)), (L - 1 - m // 2, (D // 2,))):
            bad.setdefault((b, t), tuple(cols))
    for (b, t), cols in bad.items():
        where = table[b, t // page].long(), t % page
        for c in cols:
            if kv == "e4m3":
                cache.v.view(torch.uint8)[where[0], where[1], :, c] = 0x7f
            else:
                cache.v[where[0], where[1], :, c] = (math.nan, math.inf, -math.inf)[c % 3]
    for b, entry in missing:
        table[b, entry] = -1
        keep[b, entry * page:(entry + 1) * page] = False
    ws = cake.alloc_attention_workspace(4, 2, D, DEV)
    out, lse = cake.cake_paged_chunk(q, cache, table, n, base.starts_of(new), want_lse=True, ws=ws, window=window)
    assert cake.cake_kmeans_device_status(ws) == (cake.CAKE_ERR_BAD_INDEX if missing and not window else cake.CAKE_OK)
    held = table.clamp(min=0)

    def keys_values(b, h):
        k, v = base.cached(cache, held, lens, b, h)
        return torch.where(keep[b, :lens[b], None], k, torch.zeros_like(k)), torch.where(keep[b, :lens[b], None], v, torch.zeros_like(v))
    check_around(out, lse, q, keys_values, new, lens, 2, bad, window, keep, f16=kv == "e4m3")


@pytest.mark.parametrize("D,new,lens,window", NOT_FINITE)
def test_prompt_values_that_are_not_finite_in_every_form(D, new, lens, window):
    q, k, v = base.packed(D + window, new, lens, 4, 2, D)
    at, bad = [0, lens[0], sum(lens)], {}
    for b, (m, L) in enumerate(zip(new, lens)):
        for t, cols in ((L - 1, range(D)), (L - 1 - m // 3, (3, D - 1)), (L - 1 - m // 2, (D // 2,))):
            bad.setdefault((b, t), tuple(cols))
    for (b, t), cols in bad.items():
        for c in cols:
            v[at[b] + t, :, c] = (math.nan, math.inf, -math.inf)[c % 3]
    out, lse = base.run_packed(q, k, v, new, lens, window=window)
    check_around(out, lse, q, lambda b, g: (k[at[b]:at[b + 1], g], v[at[b]:at[b + 1], g]), new, lens, 2, bad, window)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_rows_computed_again_over_a_long_context(kv):
    """As many sequences as CTAs over the same 40,000 cached tokens, the newest of which has a value that is not finite: all earlier rows of its tile are computed again."""
    B, L, n, D, page = 148, 40000, 128, 128, 64
    q, cache, table, lens = base.paged(1, [n], [L], 1, 1, D, page, kv)
    q = base.normal(base.gen(2), B * n, 1, D, std=1.2)
    where = table[0, (L - 1) // page].long(), (L - 1) % page
    if kv == "e4m3":
        cache.v.view(torch.uint8)[where[0], where[1], 0, 7] = 0x7f
    else:
        cache.v[where[0], where[1], 0, 7] = math.inf
    out, lse = base.run_chunk(q, cache, table.expand(B, -1).contiguous(), lens.expand(B).contiguous(), [n] * B)
    for b in (0, 77, B - 1):
        rows = slice(b * n, b * n + n)
        check_around(out[rows], lse[rows], q[rows], lambda _, g: base.cached(cache, table, [L], 0, g), [n], [L], 1, {(0, L - 1): (7,)}, f16=kv == "e4m3")
    assert torch.isfinite(out.view(B, n, D)[:, :-1]).all()


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 50)])
def test_what_lies_behind_a_sequence_does_not_matter(D, causal, window):
    """Padding, and a neighbour's values: NaN there gives the same bits.  Sequences whose last tile holds one key, nearly all, all; several tiles, cut items."""
    for lens in ([1, 130, 127, 128, 2, 255], [1500]):
        q, k, v = base.packed(D, lens, lens, 4, 2, D, extra=140)
        out, lse = base.run_packed(q, k, v, lens, lens, causal, window)
        k2, v2 = k.clone(), v.clone()
        k2[sum(lens):], v2[sum(lens):] = math.nan, math.inf
        again, lse2 = base.run_packed(q, k2, v2, lens, lens, causal, window)
        n = sum(lens)
        assert torch.equal(again[:n], out[:n]) and torch.equal(lse2[:n], lse[:n])
        at = 0
        for i, m in enumerate(lens):                  # every other sequence is not finite
            if i % 2:
                k2[at:at + m], v2[at:at + m] = math.nan, math.nan
            at += m
        again, lse2 = base.run_packed(q, k2, v2, lens, lens, causal, window)
        at = 0
        for i, m in enumerate(lens):
            if i % 2 == 0:
                assert torch.equal(again[at:at + m], out[at:at + m]) and torch.equal(lse2[at:at + m], lse[at:at + m])
            else:
                assert torch.isnan(again[at:at + m]).all()
            at += m


# ------------------------------------------------------------------------------------------------------- large values
def large(g, *shape):
    """Finite bf16 values of up to 3.3e38, half of them above 2^126."""
    return (base.normal(g, *shape, dtype=torch.float32) * 2.0 ** 127).clamp(-3.3e38, 3.3e38).to(BF16)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("new,lens,window", [([300, 5], [300, 5], 0), ([3], [4001], 0), ([2500], [2500], 0), ([300], [1700], 150)])
def test_finite_values_whose_sums_pass_32_bits(D, new, lens, window):
    """Their average does not: rows of whole items, of parts, and of parts that are joined."""
    q, k, v = base.packed(D + window, new, lens, 4, 2, D)
    v = large(base.gen(D), *v.shape)
    k[: lens[0] // 2] *= 0.1                          # (later keys' weights pass the first tile's by far)
    out, lse = base.run_packed(q, k, v, new, lens, window=window)
    base.check_packed(out, lse, q, k, v, new, lens, window=window)
    v[:, 1] *= 2.0 ** -9                              # beside a head whose sums do not, until its weights do
    out, lse = base.run_packed(q, k, v, new, lens, window=window)
    base.check_packed(out, lse, q, k, v, new, lens, window=window)


def test_finite_values_whose_sums_pass_32_bits_over_pages():
    new, lens = [200, 3], [330, 3000]
    q, cache, table, n = base.paged(3, new, lens, 4, 2, 128, 16, "bf16")
    cache.v.copy_(torch.where(torch.isfinite(cache.v), large(base.gen(4), *cache.v.shape), cache.v))
    out, lse = base.run_chunk(q, cache, table, n, new)
    base.check_chunk(out, lse, q, cache, table, new, lens)
    # and an infinity that some see: its column is theirs, the others are averages
    where = table[0, 320 // 16].long(), 0
    cache.v[where[0], where[1], :, 5] = math.inf
    out, lse = base.run_chunk(q, cache, table, n, new)
    check_around(out, lse, q, lambda b, g: base.cached(cache, table, lens, b, g), new, lens, 2, {(0, 320): (5,)})


# ------------------------------------------------------------------------------------------ light weights, 8-bit caches
@pytest.mark.parametrize("D,new,lens", [(64, 1, 300), (128, 200, 330), (128, 3, 4001), (256, 40, 1500)])
@pytest.mark.parametrize("where", [5, 0.6, -1])
@pytest.mark.parametrize("light", [0.5, 0.0, -1.0])
def test_light_keys_of_an_8_bit_cache(D, new, lens, where, light):
    """One key has all of the weight and values of zero; what is left are keys of 2^-28 to 2^-31 of it, all alike.  Weights hold 11 bits down to 2^-25 of the heaviest, steps of 2^-35 below:
    half a step, 2^-36, for each key, as for a decode."""
    where = int(where * lens) if 0 < where < 1 else where % lens
    new = min(new, lens - where)                      # (all of its tokens see the heavy key)
    q, cache, table, n = base.paged(2, [new], [lens], 2, 1, D, 16, "e4m3")
    g = base.gen(D)
    q.zero_()
    q[:, 0, 0], q[:, 1, 0] = 1.0, 0.5
    k = torch.zeros(lens, 1, D, device=DEV)
    k[:, 0, 0] = light
    k[where, 0, 0] = 20.0
    v = 1 + torch.rand(lens, 1, D, generator=g, device=DEV)
    v[where] = 0
    t = torch.arange(lens, device=DEV)
    at = table[0, t // 16].long(), t % 16
    cache.k.view(torch.uint8)[at], cache.v.view(torch.uint8)[at] = k.to(E4M3).view(torch.uint8), v.to(E4M3).view(torch.uint8)
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(1.0)
    out, lse = base.run_chunk(q, cache, table, n, [new], scale=1.0)
    ref, _ = cake.cake_paged_decode(q[-1:].contiguous(), cache, table, n, scale=1.0)
    kk, vv = base.cached(cache, table, [lens], 0, 0)
    want, want_lse, most, delta, _ = base.reference(q, kk, vv, 1.0, base.visible(new, lens, True, 0))
    for got, rows in ((out, slice(0, new)), (ref, slice(new - 1, new))):
        bound = (2.0 ** -11 + 2 * delta[rows] + 2 * (40 + lens / 128) * base.U)[..., None] * most[rows] + 1.01 * 2.0 ** -8 * want[rows].abs() + 1.01 * 2.0 ** -36 * vv.sum(0)
        err = (got.double() - want[rows]).abs()
        assert (err <= bound).all(), f"worst {float((err / bound).max()):.3g} bounds"
    assert ((lse.double() - want_lse).abs() <= delta + (40 + lens / 128) * base.U + 2.0 ** -22 + 2 * base.U * want_lse.abs()).all()


@pytest.mark.parametrize("D,new,lens", [(64, [40], [3000]), (128, [300, 5], [900, 2000]), (256, [20], [1500])])
@pytest.mark.parametrize("std", [0.0, 0.05, 0.4, 8.0])
def test_flat_and_steep_rows_of_an_8_bit_cache(D, new, lens, std):
    """Weights that are all alike add up to more than f16 holds although none passes it; scores that grow from tile to tile do pass it, by little and by much."""
    q, cache, table, n = base.paged(7, new, lens, 4, 2, D, 16, "e4m3", std=std)
    out, lse = base.run_chunk(q, cache, table, n, new)
    base.check_chunk(out, lse, q, cache, table, new, lens)
    q.fill_(0.25)
    for b, L in enumerate(lens):
        t = torch.arange(L, device=DEV)
        rows = ((t // 64).float() * (1 + std) * 8 / D / 0.25 / 0.02)[:, None, None].expand(L, 2, D)
        cache.k.view(torch.uint8)[table[b, t // 16].long(), t % 16] = rows.clamp(max=448).to(E4M3).contiguous().view(torch.uint8)
    out, lse = base.run_chunk(q, cache, table, n, new)
    base.check_chunk(out, lse, q, cache, table, new, lens)


# ------------------------------------------------------------------------------------------- as they are used together
@pytest.mark.parametrize("D", [64, 128, 256])
def test_pieces_of_prompts_over_an_8_bit_cache(D):
    """Norm, append and attention piece by piece: every piece against the cache's own contents in 64 bits, so that what 8 bits cost the keys and values is no excuse."""
    g = base.gen(D)
    Hq, Hkv, page, lens = 4, 2, 16, [700, 233]
    rows = base.normal(g, sum(lens), Hq + 2 * Hkv, D)
    weight = (1 + 0.2 * base.normal(g, 2, D).float()).to(BF16)
    pages = [-(-n // page) for n in lens]
    order = torch.randperm(sum(pages), device=DEV, generator=g).int()
    table = torch.full((2, max(pages)), -1, dtype=torch.int32, device=DEV)
    table[0, :pages[0]], table[1, :pages[1]] = order[:pages[0]], order[pages[0]:]
    store = [torch.zeros(sum(pages), page, Hkv, D, device=DEV).to(E4M3) for _ in range(2)]
    cache = cake.PagedCache(*store, torch.tensor([0.02, 0.03], device=DEV), torch.tensor([0.01, 0.02], device=DEV))
    ws = cake.alloc_attention_workspace(Hq, Hkv, D, DEV)
    done = [0, 0]
    for piece in ([300, 0], [1, 100], [200, 1], [0, 132], [199, 0]):
        at = torch.cat([torch.arange(d, d + n, device=DEV) for d, n in zip(done, piece)])
        owner = torch.repeat_interleave(torch.arange(2, device=DEV), torch.tensor(piece, device=DEV))
        slots = table[owner, at // page].long() * page + at % page
        x = rows[at + owner * lens[0]]
        q, _ = cake.cake_qk_norm_append(cache, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots, weight[0], weight[1], ws=ws)
        done = [d + n for d, n in zip(done, piece)]
        n = torch.tensor(done, dtype=torch.int32, device=DEV)
        out, lse = cake.cake_paged_chunk(q, cache, table, n, base.starts_of(piece), want_lse=True, ws=ws)
        base.check_chunk(out, lse, q, cache, table.clamp(min=0), piece, done)
        k, v = cake.cake_kv_read(cache, slots, ws=ws)      # what was appended is what was attended to
        for b in range(2):
            mine = owner == b
            want = [torch.stack([base.cached(cache, table.clamp(min=0), done, b, h)[i] for h in range(Hkv)], 1)[at[mine]].to(BF16) for i in range(2)]
            assert torch.equal(k[mine], want[0]) and torch.equal(v[mine], want[1])
    assert done == lens and cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


def test_scales_of_values_that_are_no_numbers():
    """They reach every row of their head that sees something, and no other head's; the rows are not computed again for it."""
    new, lens = [5, 200, 4], [3, 1500, 300]
    q, cache, table, n = base.paged(5, new, lens, 4, 2, 128, 16, "e4m3")
    want, want_lse = base.run_chunk(q, cache, table, n, new)
    cache.v_scale[1] = math.nan
    out, lse = base.run_chunk(q, cache, table, n, new)
    assert torch.equal(out[:, :2], want[:, :2]) and torch.equal(lse, want_lse)
    assert (out[:2] == 0).all() and torch.isnan(out[2:, 2:]).all()      # (the first two tokens see nothing)
