"""Attention of many tokens, norm with append and reading back as they are used: one behind the other, on streams, in graphs, from one
workspace, and at sizes whose offsets pass 32 bits."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2608_12629_b200 as cake
from tests import test_gpu_attention as base

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def example(name):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", name + ".py")
    spec = importlib.util.spec_from_file_location(name, path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("tokens", [1, 5, 777, 2000])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_chunks_add_up_to_the_prompt(tokens, eight_bit):
    """bf16: both ways round weights to bf16, the cache is exact: 2 * 2^-8 / sqrt(3) at most in norm.  8-bit: keys and values are rounded to
    e4m3 (2^-4 / sqrt(3) each; keys move the weights by scores of about that, normed queries and keys: |x| about sqrt(D) 1.44 times it)."""
    r = example("chunked_prompt").main(tokens, DEV, eight_bit=eight_bit)
    assert r["error"] < (0.5 if eight_bit else 2 * 2.0 ** -8 / math.sqrt(3)), r["error"]
    assert math.isfinite(r["lse"]) and (eight_bit or r["lse"] < 1e-4)
    if not eight_bit:
        assert torch.equal(r["keys"], r["kn"][:tokens].transpose(0, 1))      # what was appended is what is read back
    assert torch.isfinite(r["inertia"]).all()


def test_on_a_stream_of_their_own():
    lens = [300, 77]
    q, k, v = base.packed(1, lens, lens, 8, 2, 128)
    want, want_lse = base.run_packed(q, k, v, lens, lens)
    qc, cache, table, n = base.paged(2, [30, 1], [400, 90], 8, 2, 128, 16, "e4m3")
    chunk, _ = base.run_chunk(qc, cache, table, n, [30, 1])
    s = torch.cuda.Stream()
    starts, cstarts = base.starts_of(lens), base.starts_of([30, 1])
    slots = torch.arange(100, device=DEV)
    read = cake.cake_kv_read(cache, slots)
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):      # outputs and scratch are allocated for the stream, calls follow one another on it
        a, lse = cake.cake_prompt_attention(q, k, v, starts, want_lse=True, stream=s)
        b, _ = cake.cake_paged_chunk(qc, cache, table, n, cstarts, stream=s)
        c = cake.cake_kv_read(cache, slots, stream=s)
        outs.append((a, lse, b, c))
    s.synchronize()
    for a, lse, b, c in outs:
        assert torch.equal(a, want) and torch.equal(lse, want_lse) and torch.equal(b, chunk)
        assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(c, read))      # (bits: places that hold nothing are NaN)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_captured_and_replayed(kv):
    """Append, chunk and read in one graph; lengths, tables, slots and values change between replays."""
    Hq, Hkv, D, page = 8, 2, 128, 16
    q, cache, table, n = base.paged(3, [20, 1, 3], [500, 40, 3], Hq, Hkv, D, page, kv)
    g = base.gen(9)
    k, v = base.normal(g, 24, Hkv, D), base.normal(g, 24, Hkv, D)
    new, lens = [20, 1, 3], [500, 40, 3]
    starts = base.starts_of(new)

    def places(new, lens):
        owner = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(new, device=DEV))
        place = torch.cat([torch.arange(L - m, L, device=DEV) for m, L in zip(new, lens)])
        return table[owner, place // page].long() * page + place % page

    slots = places(new, lens)
    ws = cake.alloc_attention_workspace(Hq, Hkv, D, DEV)
    oq, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(24, Hq, device=DEV)
    rk, rv = torch.empty(24, Hkv, D, dtype=BF16, device=DEV), torch.empty(24, Hkv, D, dtype=BF16, device=DEV)

    def step():
        cake.cake_qk_norm_append(cache, q, k, v, slots, out_q=oq, ws=ws)
        cake.cake_paged_chunk(oq, cache, table, n, starts, out=out, out_lse=lse, ws=ws)
        cake.cake_kv_read(cache, slots, out_k=rk, out_v=rv, ws=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3):
        q.copy_(base.normal(base.gen(seed), *q.shape, std=1.2))
        k.copy_(base.normal(base.gen(seed + 10), *k.shape))
        if seed == 3:                                  # other lengths: the second sequence's chunk goes to the third
            starts.copy_(base.starts_of([20, 0, 4]))
            n[2] = 4
            slots.copy_(places([20, 0, 4], [500, 40, 4]))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (oq, out, lse, rk, rv)]
        for t in (oq, out, lse, rk, rv):
            t.fill_(3.0)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (oq, out, lse, rk, rv)))
        base.check_chunk(out, lse, oq, cache, table, [20, 1, 3] if seed < 3 else [20, 0, 4], n.tolist())
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


def test_one_workspace_for_calls_of_any_size_and_kind():
    """Back to back, without a wait: every call leaves the workspace ready for the next."""
    ws = cake.alloc_attention_workspace(8, 2, 128, DEV)
    calls = []
    for i, lens in enumerate(([2000], [1], [300, 400], [50] * 30)):
        q, k, v = base.packed(i, lens, lens, 8, 2, 128)
        calls.append((q, k, v, base.starts_of(lens), lens))
    qc, cache, table, n = base.paged(2, [30, 1], [4000, 90], 8, 2, 128, 16, "bf16")
    cs = base.starts_of([30, 1])
    got = []
    for _ in range(4):
        for q, k, v, s, _ in calls:
            got.append(cake.cake_prompt_attention(q, k, v, s, want_lse=True, ws=ws))
            got.append(cake.cake_paged_chunk(qc, cache, table, n, cs, want_lse=True, ws=ws))
    for i, (q, k, v, s, lens) in enumerate(calls):
        base.check_packed(*got[2 * i], q, k, v, lens, lens)
    base.check_chunk(*got[1], qc, cache, table, [30, 1], [4000, 90])
    for i, (out, lse) in enumerate(got):
        first = got[i % 8] if i % 2 == 0 else got[1]
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK


def test_offsets_beyond_32_bits():
    """A cache of which pages lie more than 2^32 elements apart, and an output of more than 2^31 elements."""
    if torch.cuda.mem_get_info()[0] < 40 * 2 ** 30:
        pytest.skip("needs 40 GB")
    Hkv, D, page, pages = 2, 128, 16, 3
    far = 2 ** 31 + 1024                                      # elements from page to page
    store = torch.empty(far * (pages - 1) + page * Hkv * D, dtype=BF16, device=DEV)
    kc, vc = (store.as_strided((pages, page, Hkv, D), (far - 2 ** 20, Hkv * D, D, 1), i * 2 ** 19) for i in range(2))
    g = base.gen(1)
    k, v = base.normal(g, 40, Hkv, D), base.normal(g, 40, Hkv, D)
    cache = cake.PagedCache(kc, vc)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
    t = torch.arange(40, device=DEV)
    slots = table[0, t // page].long() * page + t % page
    q = base.normal(g, 40, 4, D, std=1.2)
    oq, ok = cake.cake_qk_norm_append(cache, q, k, v, slots, want_k=True)
    back = cake.cake_kv_read(cache, slots)
    assert torch.equal(back[0], ok) and torch.equal(back[1], v)
    n = torch.tensor([40], dtype=torch.int32, device=DEV)
    out, lse = base.run_chunk(oq, cache, table, n, [40])
    ref, ref_lse = base.run_packed(oq, ok, v, [40], [40])
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    del store, kc, vc, cache
    torch.cuda.empty_cache()
    T, Hq, D = 2 ** 17 + 5, 128, 128                          # 2^31 elements of queries and as many of the output
    q = torch.zeros(T, Hq, D, dtype=BF16, device=DEV)
    k, v = base.normal(g, T, 1, D), base.normal(g, T, 1, D)
    starts = torch.arange(0, T + 1, 5, dtype=torch.int32, device=DEV)
    starts = torch.cat([starts, starts.new_tensor([T])])
    out, lse = cake.cake_prompt_attention(q, k, v, starts, want_lse=True)
    for b in (0, len(starts) - 3, len(starts) - 2):           # queries of zero: means of the values so far
        s0, s1 = int(starts[b]), int(starts[b + 1])
        want = v[s0:s1, 0].double().cumsum(0) / torch.arange(1, s1 - s0 + 1, device=DEV)[:, None]
        got = out[s0:s1].double()
        assert ((got - want[:, None]).abs() <= 2.0 ** -7 * (want.abs() + 1)[:, None]).all()
        assert (lse[s0:s1].double() - torch.arange(1, s1 - s0 + 1, device=DEV).double().log()[:, None]).abs().max() < 1e-6


def test_host_threads_at_once():
    """First calls on a device from several threads, each with a stream and a workspace of its own."""
    import threading
    lens = [200, 3]
    q, k, v = base.packed(5, lens, lens, 4, 2, 96)
    want, _ = base.run_packed(q, k, v, lens, lens)
    starts = base.starts_of(lens)
    torch.cuda.synchronize()
    got, errors = [None] * 4, []

    def work(i):
        try:
            s = torch.cuda.Stream()
            for _ in range(20):
                got[i], _ = cake.cake_prompt_attention(q, k, v, starts, stream=s)
            s.synchronize()
        except Exception as e:      # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and all(torch.equal(x, want) for x in got)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_outputs_at_every_allowed_alignment(D):
    """out is 16-byte aligned: a buffer 16 bytes behind a multiple of 32 gets the same bits, and nothing beside it is touched."""
    lens = [130, 2500, 7]
    q, k, v = base.packed(5, lens, lens, 4, 2, D)
    want, _ = base.run_packed(q, k, v, lens, lens)
    room = torch.full((q.numel() + 32,), 7.0, dtype=BF16, device=DEV)
    out = room[8:8 + q.numel()].view(sum(lens), 4, D)
    assert out.data_ptr() % 32 == 16
    cake.cake_prompt_attention(q, k, v, base.starts_of(lens), out=out)
    assert torch.equal(out, want)
    assert (room[:8] == 7).all() and (room[8 + q.numel():] == 7).all()


def test_sequences_of_one_row_tile_beside_larger_ones():
    """Items of one row tile count half when work is shared out: long rows of single tokens beside pieces of prompts, and prompts whose last
    block is one tile, in windows and without."""
    new, lens = [1, 900, 1, 65, 1, 32, 1], [3900, 2100, 5000, 65, 1, 4000, 129]
    for window in (0, 777):
        for kv in ("bf16", "e4m3"):
            q, cache, table, n = base.paged(7, new, lens, 8, 2, 128, 16, kv)
            out, lse = base.run_chunk(q, cache, table, n, new, window=window)
            base.check_chunk(out, lse, q, cache, table, new, lens, window=window)
        q, k, v = base.packed(8, new, lens, 8, 2, 64)
        out, lse = base.run_packed(q, k, v, new, lens, window=window)
        base.check_packed(out, lse, q, k, v, new, lens, window=window)
    out, lse = base.run_packed(q, k, v, new, lens, causal=False)
    base.check_packed(out, lse, q, k, v, new, lens, causal=False)


def test_scales_of_zero_weigh_all_visible_keys_alike():
    """A head whose keys' scale is zero has scores of zero: the mean of the values that a token sees, log of their number, masked keys left out."""
    new, lens = [3, 140], [50, 300]
    q, cache, table, n = base.paged(11, new, lens, 4, 2, 128, 16, "e4m3")
    cache.k_scale[0] = 0.0
    out, lse = base.run_chunk(q, cache, table, n, new, window=100)
    base.check_chunk(out, lse, q, cache, table, new, lens, window=100)
    q[5:40] *= 2.0 ** -125      # and queries next to nothing
    out, lse = base.run_chunk(q, cache, table, n, new)
    base.check_chunk(out, lse, q, cache, table, new, lens)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("window", [0, 150, 300])
def test_pages_out_of_range_inside_windows_and_pieces(kv, window):
    """The second row tile of an item may begin behind the first one's first tile of keys: it sees its own tiles' missing pages."""
    page, new, lens = 16, [900, 70], [2000, 1500]
    q, cache, table, n = base.paged(13, new, lens, 4, 1, 128, page, kv)
    keep = torch.ones(2, 2000, dtype=torch.bool, device=DEV)
    for b, entry in ((0, 69), (0, 75), (0, 90), (0, 117), (1, 81), (1, 92)):
        table[b, entry] = -1
        keep[b, entry * page:(entry + 1) * page] = False
    ws = cake.alloc_attention_workspace(4, 1, 128, DEV)
    out, lse = cake.cake_paged_chunk(q, cache, table, n, base.starts_of(new), want_lse=True, ws=ws, window=window)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_ERR_BAD_INDEX
    table.clamp_(min=0)
    base.check(out, lse, q, lambda b, g: tuple(torch.nan_to_num(x) for x in base.cached(cache, table, lens, b, g)), new, lens, 1, 128 ** -0.5, True, window,
               f16=kv == "e4m3", keep=lambda b, g: keep[b, :lens[b]])
