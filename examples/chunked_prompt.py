"""A prompt through one attention layer of a serving program, at once and in chunks behind a cached prefix.

    query/key/value projection -> norm of each head + rotation + paged cache -> attention
      at once:    the prompt's keys and values as they come (packed prompts)
      in chunks:  each chunk over the pages that hold the ones before it; the last tokens one by one are chunks of one
    and the cached keys read back as one matrix per head, as the clustering takes them

Run it with `python examples/chunked_prompt.py [tokens]` on a B200: it prints how far the two ways are apart, over a bf16 cache and over an
8-bit one.  Weights and hidden states are synthetic.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_12629_b200 as cake  # noqa: E402
from paper_2608_12629_b200 import inputs  # noqa: E402

HQ, HKV, D, PAGE = 8, 2, 128, 16


def rotary_table(longest, device):
    angle = torch.arange(longest, device=device, dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(0, D, 2, device=device, dtype=torch.float64) / D)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def main(tokens=2000, device="cuda:0", seed=0, chunk=512, eight_bit=False):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    # two prompts, packed: what a projection of them holds, queries, keys and values side by side
    lens = [tokens, max(1, tokens // 3)]
    starts = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device=device)
    rows = torch.randn(sum(lens), HQ + 2 * HKV, D, generator=g, device=device).bfloat16()
    q, k, v = rows[:, :HQ], rows[:, HQ:HQ + HKV], rows[:, HQ + HKV:]
    weight = (1 + 0.2 * torch.randn(2, D, generator=g, device=device)).bfloat16()
    pages = [-(-n // PAGE) for n in lens]
    order = torch.randperm(sum(pages), generator=g, device=device)
    table = torch.full((2, max(pages)), -1, dtype=torch.int32, device=device)
    table[0, :pages[0]], table[1, :pages[1]] = order[:pages[0]].int(), order[pages[0]:].int()
    position = torch.cat([torch.arange(n, device=device) for n in lens])
    owner = torch.repeat_interleave(torch.arange(2, device=device), torch.tensor(lens, device=device))
    slots = table[owner, position // PAGE].long() * PAGE + position % PAGE
    shape, dtype = (sum(pages), PAGE, HKV, D), torch.float8_e4m3fn if eight_bit else torch.bfloat16
    scale = torch.full((HKV,), 0.02, device=device) if eight_bit else None
    cache = cake.PagedCache(torch.zeros(shape, device=device).to(dtype), torch.zeros(shape, device=device).to(dtype), scale, scale)
    ws = cake.alloc_attention_workspace(HQ, HKV, D, device)

    # at once
    qn, kn = cake.cake_qk_norm_append(cache, q, k, v, slots, weight[0], weight[1], position.int(), rotary_table(max(lens), device), want_k=True, ws=ws)
    whole, whole_lse = cake.cake_prompt_attention(qn, kn, v, starts, want_lse=True, ws=ws)

    # in chunks: both sequences' next tokens in one call, the shorter one's until it ends
    out, lse = torch.empty_like(whole), torch.empty_like(whole_lse)
    done = 0
    while done < max(lens):
        size = chunk if done + chunk < max(lens) - 2 else 1 if done >= max(lens) - 2 else max(lens) - 2 - done
        new = [max(0, min(n, done + size) - done) for n in lens]
        picked = torch.cat([torch.arange(done, done + n, device=device) + int(s) for n, s in zip(new, (0, lens[0]))])
        part, part_lse = cake.cake_paged_chunk(qn[picked], cache, table, torch.tensor([min(n, done + size) for n in lens], dtype=torch.int32, device=device),
                                               torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device=device), want_lse=True, ws=ws)
        out[picked], lse[picked] = part, part_lse
        done += size

    # a head's cached keys as one matrix: what the clustering takes
    keys, _ = cake.cake_kv_read(cache, slots[:lens[0]], by_head=True, want_v=False, ws=ws)
    clusters = min(16, lens[0])
    found = cake.cake_kmeans_lloyd(keys[0], inputs.sample_init(keys[0], clusters, seed), 3)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK
    error = ((out.float() - whole.float()).norm() / whole.float().norm()).item()
    return dict(tokens=sum(lens), error=error, lse=(lse - whole_lse).abs().max().item(), keys=keys, kn=kn, inertia=found.inertia)


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 2000
    for eight_bit in (False, True):
        r = main(n, eight_bit=eight_bit)
        print(f"{r['tokens']} tokens, {'8-bit' if eight_bit else 'bf16'} cache: chunks and the whole prompt {100 * r['error']:.2f} % apart")
