"""One attention layer of a serving step over a cache whose keys are clustered.

    hidden states -> norm + 8-bit -> query/key/value projection -> rotation + paged cache
    cached keys -> Lloyd (clusters per head) -> nearest clusters of the query -> attention over their tokens alone
    attention output -> 8-bit -> output projection -> norm + residual of the next layer

Every step is a call of this library; PyTorch holds the memory and builds the list of the selected tokens.  Run it with
`python examples/clustered_decode.py [tokens]` on a B200: it prints how many tokens were read and how much of the full attention's
mass and output they carry.  Weights and hidden states are synthetic (a mixture: tokens of one component have similar keys).
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_12629_b200 as cake  # noqa: E402
from paper_2608_12629_b200 import inputs  # noqa: E402

HIDDEN, HQ, HKV, D, PAGE = 1024, 8, 2, 64, 16
CLUSTERS, ITERS, NEAREST, RECENT = 64, 6, 4, 64
ROT = 16                       # rotate a quarter of each head, so that clusters gather tokens from all positions


def quantise_weights(w: torch.Tensor):
    """[N,K] fp32 -> e4m3 and one scale per 128 x 128 block (done once, when a model is loaded)."""
    n, k = w.shape
    nb, kb = -(-n // 128), -(-k // 128)
    padded = torch.zeros(nb * 128, kb * 128, device=w.device)
    padded[:n, :k] = w
    blocks = padded.view(nb, 128, kb, 128)
    scale = (blocks.abs().amax((1, 3)) / 448).clamp(min=1e-12)
    q = (blocks / scale[:, None, :, None]).reshape(nb * 128, kb * 128)[:n, :k].contiguous().to(torch.float8_e4m3fn)
    return q, scale.contiguous()


class Layer:
    def __init__(self, device, seed=0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        wk = torch.randn(HKV, D, HIDDEN, generator=g, device=device) / HIDDEN ** 0.5
        # a query looks for tokens like its own: each query head is its key head, sharpened
        wq = (1.3 * wk)[:, None].expand(HKV, HQ // HKV, D, HIDDEN).reshape(HQ * D, HIDDEN)
        wv = torch.randn(HKV * D, HIDDEN, generator=g, device=device) / HIDDEN ** 0.5
        self.qkv = quantise_weights(torch.cat([wq, wk.reshape(HKV * D, HIDDEN), wv]))
        self.out = quantise_weights(torch.randn(HIDDEN, HQ * D, generator=g, device=device) / (HQ * D) ** 0.5)
        self.norm = torch.ones(HIDDEN, dtype=torch.bfloat16, device=device)

    def project(self, hidden, residual=None):
        """hidden (+ residual) -> q, k, v as views of one projection, and the residual stream."""
        x, scale, _, stream = cake.cake_rmsnorm_quant(hidden, self.norm, residual, want_residual=True)
        rows = cake.cake_gemm_fp8(x, scale, *self.qkv).view(-1, HQ + 2 * HKV, D)
        return rows[:, :HQ], rows[:, HQ:HQ + HKV], rows[:, HQ + HKV:], stream

    def finish(self, attended, stream):
        """Attention output -> output projection; the next layer's norm adds it to the residual stream."""
        x, scale, _, _ = cake.cake_rmsnorm_quant(attended.view(-1, HQ * D), flags=cake.CAKE_RMSNORM_NONE)
        return cake.cake_rmsnorm_quant(cake.cake_gemm_fp8(x, scale, *self.out), self.norm, stream, want_q=False, want_y=True)[2]


def rotary_table(longest, device):
    angle = torch.arange(longest, device=device, dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(0, ROT, 2, device=device, dtype=torch.float64) / ROT)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def main(tokens=4096, device="cuda:0", seed=0):
    layer = Layer(device, seed)
    pages = -(-(tokens + 1) // PAGE)
    k_cache, v_cache = (torch.zeros(pages, PAGE, HKV, D, dtype=torch.bfloat16, device=device) for _ in range(2))
    cache = cake.PagedCache(k_cache, v_cache)
    table = rotary_table(tokens + 1, device)
    ws = cake.alloc_decode_workspace(1, HQ, HKV, D, device)

    # the prompt: all tokens but the last at once
    hidden, _ = inputs.gaussian_mixture(tokens + 1, HIDDEN, 32, 1.0, 0.4, seed + 3)
    hidden = hidden.to(device)
    # pages are handed out in any order, filled from their start
    slots = (torch.randperm(pages, device=device)[:, None] * PAGE + torch.arange(PAGE, device=device)).view(-1)[:tokens + 1].contiguous()
    position = torch.arange(tokens + 1, dtype=torch.int32, device=device)
    _, k, v, _ = layer.project(hidden[:tokens])
    cake.cake_kv_append(cache, k, v, slots[:tokens], position[:tokens], table, ws=ws)

    # clusters of each head's cached keys
    flat = k_cache.view(-1, HKV, D)
    found = []
    for h in range(HKV):
        keys = flat[slots[:tokens], h].contiguous()
        found.append(cake.cake_kmeans_lloyd(keys, inputs.sample_init(keys, CLUSTERS, seed + h), ITERS))

    # a decode step: the new token into the cache, its clusters, attention over their tokens and the most recent ones
    q, k, v, stream = layer.project(hidden[tokens:])
    q = cake.cake_kv_append(cache, k, v, slots[tokens:], position[tokens:], table, q=q, ws=ws)
    group = HQ // HKV
    chosen = []
    for h in range(HKV):
        near, _ = cake.cake_knn_search(q[0, h * group:(h + 1) * group].contiguous(), found[h].C_bf16, NEAREST)
        keep = torch.zeros(CLUSTERS, dtype=torch.bool, device=device)
        keep[near.long().view(-1)] = True
        picked = keep[found[h].idx.long()]
        picked[max(0, tokens - RECENT):] = True
        chosen.append(torch.cat([slots[:tokens][picked], slots[tokens:]]))
    lens = torch.tensor([[c.numel() for c in chosen]], dtype=torch.int32, device=device)
    per_head = torch.full((1, HKV, int(lens.max())), -1, dtype=torch.int32, device=device)
    for h, c in enumerate(chosen):
        per_head[0, h, :c.numel()] = c.int()
    # the same memory as pages of one token: a table per key-value head names tokens instead of pages
    by_token = cake.PagedCache(k_cache.view(-1, 1, HKV, D), v_cache.view(-1, 1, HKV, D))
    out, lse = cake.cake_paged_decode(q, by_token, per_head, lens, want_lse=True, ws=ws)
    result = layer.finish(out, stream)

    # against attention over the whole cache
    page_table = (slots[::PAGE] // PAGE).int()[None].contiguous()
    full, full_lse = cake.cake_paged_decode(q, cache, page_table, torch.tensor([tokens + 1], dtype=torch.int32, device=device), want_lse=True, ws=ws)
    assert cake.cake_kmeans_device_status(ws) == cake.CAKE_OK
    error = ((out.float() - full.float()).norm() / full.float().norm()).item()
    return dict(tokens=tokens + 1, read=lens.float().mean().item(), mass=(lse - full_lse).exp().min().item(), error=error, result=result)


if __name__ == "__main__":
    r = main(int(sys.argv[1]) if len(sys.argv) > 1 else 4096)
    print(f"{r['tokens']} cached tokens, {r['read']:.0f} read per head: at least {100 * r['mass']:.1f} % of the attention mass, "
          f"output off by {100 * r['error']:.1f} %")
