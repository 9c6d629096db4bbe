"""Attention of many tokens at the edges of its range, against a plain implementation in 64 bits: scales that are no numbers or next to nothing.

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
