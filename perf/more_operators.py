"""Cases and plain forms of the serving operators for many tokens: prompt_attention, paged_chunk, qk_norm_append, kv_read.

Where `own` is false, `run` computes an operator with elementary torch operations in 32 bits, rounded once at the end; where it
is true, it calls this library.  `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
DEV = "cuda"
EPS = 1e-6
INF = math.inf


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one short prompt: the first token's latency
        dict(name="prompt-short", op="prompt", B=1, T=201, Hq=32, Hkv=8, D=128, causal=True, window=0),
        # a batch of ragged prompts, packed
        dict(name="prompt-packed", op="prompt", B=8, T=8192, Hq=32, Hkv=8, D=128, causal=True, window=0),
        # one long prompt: tensor-core bound
        dict(name="prompt-long", op="prompt", B=1, T=16384, Hq=32, Hkv=8, D=128, causal=True, window=0),
        # layers with a sliding window and narrow heads, a key-value head to each query head
        dict(name="prompt-window", op="prompt", B=4, T=12001, Hq=16, Hkv=16, D=64, causal=True, window=1024),
        # four proposed tokens a sequence to be checked against its cache: bound by reading the cache
        dict(name="chunk-verify", op="chunk", B=16, T=64, Hq=32, Hkv=8, D=128, page=16, kv="bf16", longest=4097, window=0),
        # a step that mixes sequences with one new token and sequences with a piece of their prompt
        dict(name="chunk-mixed", op="chunk", B=24, T=3001, Hq=32, Hkv=8, D=128, page=64, kv="bf16", longest=6000, window=0),
        # two long contexts in an 8-bit cache, the next piece of each prompt
        dict(name="chunk-long-e4m3", op="chunk", B=2, T=2048, Hq=64, Hkv=8, D=128, page=64, kv="e4m3", longest=32768, window=0),
        # a decode step of 16 sequences
        dict(name="qknorm-16", op="qknorm", T=16, Hq=32, Hkv=8, D=128, rot=128, pairs=False, page=16, kv="bf16", pool=65536, dense_k=False),
        # a packed prompt, whose keys go to the prompt's own attention as well as to the cache
        dict(name="qknorm-prompt", op="qknorm", T=16001, Hq=32, Hkv=8, D=128, rot=128, pairs=False, page=16, kv="bf16", pool=65536, dense_k=True),
        # a prompt into an 8-bit cache, wide heads that turn in part
        dict(name="qknorm-e4m3", op="qknorm", T=5000, Hq=16, Hkv=4, D=256, rot=64, pairs=False, page=64, kv="e4m3", pool=65536, dense_k=False),
        # one sequence's keys for the clustering, a matrix for each head
        dict(name="read-one", op="read", N=777, Hkv=8, D=128, page=16, kv="bf16", pool=65536, by_head=True, values=False),
        # a long prefix from an 8-bit cache, keys and values
        dict(name="read-prefix", op="read", N=100001, Hkv=8, D=128, page=64, kv="e4m3", pool=262144, by_head=False, values=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _heads(rng):
    Hkv = rng.choice([1, 2, 4, 8, 16])
    return Hkv * rng.choice([1, 2, 3, 4, 5, 6, 8] if Hkv < 8 else [1, 2, 4, 8] if Hkv == 8 else [1, 2, 3]), Hkv


def draw(rng):
    op = rng.choice(["prompt", "prompt", "chunk", "chunk", "qknorm", "read"])
    Hq, Hkv = _heads(rng)
    D = rng.choice([64, 96, 128, 128, 256])
    if op == "prompt":
        B = _log(rng, 1, 16)
        # the largest listed case's work, and a plain form of a few GB a key-value head: B (2 T / B)^2 scores for each query head
        most = min(16384, int((2.0 ** 40 / (2 * Hq * D) * B / 4) ** 0.5), int((2.0 ** 29 * B / 4 / (Hq // Hkv)) ** 0.5))
        T = max(B, _log(rng, 16, max(16, most)))
        window = rng.choice([0, 0, 0, max(1, T // B // 3)])
        return dict(op=op, B=B, T=T, Hq=Hq, Hkv=Hkv, D=D, causal=window > 0 or rng.random() < 0.8, window=window)
    page = rng.choice([1, 8, 16, 16, 32, 64, 100, 128])
    kv = rng.choice(["bf16", "bf16", "e4m3"])
    if op == "chunk":
        B = _log(rng, 1, 48)
        width = Hkv * D * (4 if kv == "bf16" else 2)                              # bytes of one token's keys and values
        cached = _log(rng, 32 * B, max(32 * B, min(2 ** 29 // width, 131072)))    # over the whole batch
        longest = max(2, 2 * cached // B)
        most = min(4096, int(2.0 ** 39 / (2 * Hq * D * longest)), int(2.0 ** 29 / 2 / (Hq // Hkv) / longest), B * longest // 20)
        T = max(B, _log(rng, B, max(B, most)))
        return dict(op=op, B=B, T=T, Hq=Hq, Hkv=Hkv, D=D, page=page, kv=kv, longest=longest,
                    window=rng.choice([0, 0, 0, max(1, longest // 3)]))
    if op == "qknorm":
        return dict(op=op, T=_log(rng, 1, 16384 * 48 * 128 // ((Hq + 2 * Hkv) * D) // 2), Hq=Hq, Hkv=Hkv, D=D, rot=rng.choice([D, D, D // 2, 0]),
                    pairs=rng.random() < 0.4, page=page, kv=kv, pool=131072 // max(1, Hkv * D // 512), dense_k=rng.random() < 0.4)
    return dict(op=op, N=_log(rng, 1, 2 ** 26 // (Hkv * D)), Hkv=Hkv, D=D, page=page, kv=kv, pool=2 ** 27 // (Hkv * D),
                by_head=rng.random() < 0.5, values=rng.random() < 0.6)


# ------------------------------------------------------------------------------------------------------------ inputs
def _split(total, n):
    """`total` in n parts of at least one, ragged and fixed by the numbers: from about a quarter to twice the mean."""
    weights = [4 + (i * 7 % n) * 28 // n for i in range(n)]
    parts = [max(1, (total - n) * w // sum(weights) + 1) for w in weights]
    parts[-1] += total - sum(parts)
    return parts


def _chunks(case):
    """(new tokens, tokens with them) of each sequence: every other one has a single new token where there is a mixture."""
    B, T, L = case["B"], case["T"], case["longest"]
    single = T >= 8 * B and B > 2
    few = [i for i in range(B) if single and i % 2]
    many = iter(_split(T - len(few), B - len(few)))
    new = [1 if i in few else next(many) for i in range(B)]
    return new, [n + max(0, L - n - (i * 5 % B) * (L - L // 8) // B) for i, n in enumerate(new)]


def _normal(gen, *shape, std=1.0, dtype=torch.bfloat16):
    out = torch.empty(*shape, dtype=dtype, device=DEV)
    return out.normal_(0.0, std, generator=gen)


def _e4m3(gen, *shape, std):
    out = torch.empty(*shape, dtype=E4M3, device=DEV)
    step = max(1, 2 ** 28 // max(1, out[0].numel()))
    for a in range(0, shape[0], step):      # (piece by piece: the bf16 copy is as large as two caches)
        out[a:a + step] = _normal(gen, *out[a:a + step].shape, std=std).to(E4M3)
    return out


def _uniform(gen, *shape, lo, hi):
    return torch.empty(*shape, dtype=torch.float32, device=DEV).uniform_(lo, hi, generator=gen)


def _starts(lens):
    return torch.tensor([0] + lens, dtype=torch.int64).cumsum(0).to(torch.int32).to(DEV)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, Hkv, D = case["op"], case["Hkv"], case["D"]
    if op == "prompt":
        # one projection's output holds q, k and v side by side; logits of a spread of about 1.5
        qkv = _normal(gen, case["T"], case["Hq"] + 2 * Hkv, D, std=1.22)
        Hq = case["Hq"]
        lens = _split(case["T"], case["B"])
        return dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], starts=_starts(lens), new=lens, lens=lens)
    page = case["page"]
    e = case["kv"] == "e4m3"
    scales = dict(ks=_uniform(gen, Hkv, lo=0.01, hi=0.025) if e else None, vs=_uniform(gen, Hkv, lo=0.01, hi=0.025) if e else None)

    def cache(pages):
        return _e4m3(gen, pages, page, Hkv, D, std=60.0) if e else _normal(gen, pages, page, Hkv, D)
    if op == "chunk":
        new, lens = _chunks(case)
        need = torch.tensor([-(-n // page) for n in lens])
        width, pages = int(need.max()), int(need.sum()) + 3
        order = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)      # pages are handed out in random order
        first = torch.cat([torch.zeros(1, dtype=torch.int64), need.cumsum(0)[:-1]])
        at = (first[:, None] + torch.arange(width)[None, :]).clamp_(max=pages - 1).to(DEV)
        table = order[at]
        table[torch.arange(width)[None, :].to(DEV) >= need.to(DEV)[:, None]] = -1
        return dict(q=_normal(gen, case["T"], case["Hq"], D, std=1.5), kc=cache(pages), vc=cache(pages), table=table, starts=_starts(new),
                    seq_lens=torch.tensor(lens, dtype=torch.int32).to(DEV), new=new, lens=lens, **scales)
    pages = -(-case["pool"] // page)
    if op == "qknorm":
        T, Hq, rot = case["T"], case["Hq"], case["rot"]
        longest = 32768
        freq = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1))
        angle = torch.arange(longest, device=DEV, dtype=torch.float64)[:, None] * freq[None, :]
        kc, vc = (torch.zeros(pages, page, Hkv, D, dtype=E4M3 if e else torch.bfloat16, device=DEV) for _ in range(2))
        slots = torch.randperm(pages * page, device=DEV, generator=gen)[:T].clone()
        slots[5::97] = -1                                   # padding rows of a batch: nothing is written for them
        qkv = _normal(gen, T, Hq + 2 * Hkv, D, std=2.0)
        qkv[:, :, :: max(1, D // 5)] *= 8.0                 # a few outlier features, as projections have
        return dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], kc=kc, vc=vc, slots=slots,
                    wq=_normal(gen, D, std=0.2) + 1.0, wk=_normal(gen, D, std=0.2) + 1.0,
                    pos=torch.randint(0, longest, (T,), device=DEV, generator=gen, dtype=torch.int32),
                    table=torch.cat([angle.cos(), angle.sin()], 1).float() if rot else None, **scales)
    # pages of one sequence, in the order of its tokens
    order = torch.randperm(pages, device=DEV, generator=gen)
    t = torch.arange(case["N"], device=DEV)
    return dict(kc=cache(pages), vc=cache(pages), slots=order[t // page] * page + t % page, **scales)


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    if own:     # what a serving program keeps between steps: the cache's handle, the workspace, output buffers
        import paper_2608_12629_b200 as cake
        s["cake"] = cake
        op, Hkv, D = case["op"], case["Hkv"], case["D"]
        if op != "prompt":
            s["cache"] = cake.PagedCache(s["kc"], s["vc"], s["ks"], s["vs"])
        if op in ("prompt", "chunk"):
            s["out"] = torch.empty(case["T"], case["Hq"], D, dtype=torch.bfloat16, device=DEV)
            s["lse"] = torch.empty(case["T"], case["Hq"], dtype=torch.float32, device=DEV)
            s["buf"] = cake.alloc_attention_workspace(case["Hq"], Hkv, D, DEV)
        elif op == "qknorm":
            s["out_q"] = torch.empty(case["T"], case["Hq"], D, dtype=torch.bfloat16, device=DEV)
            s["out_k"] = torch.empty(case["T"], Hkv, D, dtype=torch.bfloat16, device=DEV) if case["dense_k"] else None
            s["buf"] = cake.alloc_append_workspace(DEV)
        else:
            shape = (Hkv, case["N"], D) if case["by_head"] else (case["N"], Hkv, D)
            s["out_k"], s["out_v"] = (torch.empty(*shape, dtype=torch.bfloat16, device=DEV) if wanted else None
                                      for wanted in (True, case["values"]))
            s["buf"] = cake.alloc_append_workspace(DEV)
    return s


# ------------------------------------------------------------------------------------------------------------ passes
def run(s):
    return (_run_own if own else _run_plain)(s, s["case"])


def _run_own(s, c):
    cake, op = s["cake"], c["op"]
    if op == "prompt":
        out, lse = cake.cake_prompt_attention(s["q"], s["k"], s["v"], s["starts"], causal=c["causal"], window=c["window"], out=s["out"],
                                              out_lse=s["lse"], ws=s["buf"])
        return dict(out=out, lse=lse)
    if op == "chunk":
        out, lse = cake.cake_paged_chunk(s["q"], s["cache"], s["table"], s["seq_lens"], s["starts"], window=c["window"], out=s["out"],
                                         out_lse=s["lse"], ws=s["buf"])
        return dict(out=out, lse=lse)
    if op == "qknorm":
        q, k = cake.cake_qk_norm_append(s["cache"], s["q"], s["k"], s["v"], s["slots"], s["wq"], s["wk"], s["pos"] if c["rot"] else None,
                                        s["table"], eps=EPS, interleaved=c["pairs"], out_q=s["out_q"], out_k=s["out_k"], ws=s["buf"])
        return dict(q=q, k=k, k_cache=s["kc"], v_cache=s["vc"])
    k, v = cake.cake_kv_read(s["cache"], s["slots"], out_k=s["out_k"], out_v=s["out_v"], by_head=c["by_head"], want_v=c["values"], ws=s["buf"])
    return dict(k=k, v=v)


def _run_plain(s, c):
    return globals()["_plain_" + c["op"]](s, c)


def _attention(q, heads, starts, lens, c, ks=None, vs=None):
    """Attention of packed queries, every sequence padded to the longest; heads(g) gives the padded keys and values [B, L, D] of a
    key-value head (one after the other: all scores at once are tens of GB)."""
    T, Hq, D = q.shape
    G = Hq // c["Hkv"]
    new = (starts[1:] - starts[:-1]).long()
    n = int(max(s for s in c["new"]))
    i = torch.arange(n, device=DEV)
    at = (starts[:-1].long()[:, None] + i).clamp(max=T - 1)                    # [B, n]
    real = i < new[:, None]
    out = torch.empty(T, Hq, D, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(T, Hq, dtype=torch.float32, device=DEV)
    rows = at[real]
    for g in range(c["Hkv"]):
        k, v = heads(g)
        t = torch.arange(k.shape[1], device=DEV)
        last = (lens[:, None] - new[:, None] + i)[:, :, None]                   # a token's own position
        seen = t < lens[:, None, None]
        if c.get("causal", True):
            seen = seen & (t <= last)
        if c["window"]:
            seen = seen & (t > last - c["window"])
        scale = 1.0 / math.sqrt(D) * (1.0 if ks is None else ks[g])
        x = (q[at, g * G:(g + 1) * G].float() * scale).transpose(1, 2) @ k[:, None].transpose(2, 3)     # [B, G, n, L]
        x.masked_fill_(~seen[:, None], -INF)
        m = x.amax(3, keepdim=True).clamp(min=-1e30)
        x.sub_(m).exp_()
        total = x.sum(3, keepdim=True)
        o = (x @ v[:, None]) / total * (1.0 if vs is None else vs[g])
        out[rows, g * G:(g + 1) * G] = o.transpose(1, 2)[real].to(torch.bfloat16)
        lse[rows, g * G:(g + 1) * G] = (m + torch.log(total))[..., 0].transpose(1, 2)[real]
        del k, v, x, o
    return dict(out=out, lse=lse)


def _plain_prompt(s, c):
    starts = s["starts"]
    lens = (starts[1:] - starts[:-1]).long()
    at = (starts[:-1].long()[:, None] + torch.arange(max(s["lens"]), device=DEV)).clamp(max=c["T"] - 1)
    return _attention(s["q"], lambda g: (s["k"][at, g].float(), s["v"][at, g].float()), starts, lens, dict(c, new=s["new"]))


def _plain_chunk(s, c):
    table = s["table"].clamp(min=0).long()

    def heads(g):
        return tuple((cache[:, :, g].view(torch.uint8)[table].view(E4M3) if cache.dtype == E4M3 else cache[:, :, g][table]).flatten(1, 2).float()
                     for cache in (s["kc"], s["vc"]))
    return _attention(s["q"], heads, s["starts"], s["seq_lens"].long(), dict(c, new=s["new"]), s["ks"], s["vs"])


def _rotate(x, cos, sin, rot, pairs):
    """x [T, heads, D]; cos, sin [T, rot / 2]."""
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., :rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if pairs else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_qknorm(s, c):
    made = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * w.float()
        if c["rot"]:
            x = _rotate(x, *s["table"][s["pos"].long()].chunk(2, 1), c["rot"], c["pairs"])
        made.append(x)
    q, k = made
    v = s["v"].float()
    dense = k.to(torch.bfloat16) if c["dense_k"] else None
    if s["ks"] is not None:
        k = (k / s["ks"][:, None]).clamp(-E4M3_MAX, E4M3_MAX)
        v = (v / s["vs"][:, None]).clamp(-E4M3_MAX, E4M3_MAX)
    kept = s["slots"] >= 0
    for cache, new in ((s["kc"], k), (s["vc"], v)):
        byte = cache.element_size() == 1
        new = new.to(cache.dtype)
        (cache.view(torch.uint8) if byte else cache).view(-1, c["Hkv"], c["D"])[s["slots"][kept]] = (new.view(torch.uint8) if byte else new)[kept]
    return dict(q=q.to(torch.bfloat16), k=dense, k_cache=s["kc"], v_cache=s["vc"])


def _plain_read(s, c):
    def rows(cache, scale):
        flat = cache.view(-1, c["Hkv"], c["D"])
        x = (flat.view(torch.uint8)[s["slots"]].view(E4M3) if cache.dtype == E4M3 else flat[s["slots"]]).float()
        if scale is not None:
            x = x * scale[:, None]
        x = x.to(torch.bfloat16)
        return x.transpose(0, 1).contiguous() if c["by_head"] else x
    return dict(k=rows(s["kc"], s["ks"]), v=rows(s["vc"], s["vs"]) if c["values"] else None)


# ------------------------------------------------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    return globals()["_exact_" + case["op"]](_inputs(case, seed), case)


def _exact_sequence(q, k, v, scale, causal, window):
    """q [n, G, D], k and v [L, D] of one sequence and key-value head, in 64 bits: the last n of the L positions ask."""
    n, L = q.shape[0], k.shape[0]
    outs, sums = [], []
    step = max(1, 2 ** 27 // (q.shape[1] * L))
    for a in range(0, n, step):
        z = torch.einsum("igd,td->igt", q[a:a + step], k) * scale
        hidden = torch.zeros(z.shape[0], L, dtype=torch.bool, device=DEV)
        own_place = L - n + a + torch.arange(z.shape[0], device=DEV)[:, None]
        away = own_place - torch.arange(L, device=DEV)[None, :]           # how far a key lies behind
        if causal:
            hidden |= away < 0
        if window:
            hidden |= away >= window
        z[hidden[:, None, :].expand_as(z)] = -INF
        s = torch.logsumexp(z, 2)
        outs.append(torch.einsum("igt,td->igd", (z - s[..., None]).exp(), v))
        sums.append(s)
    return torch.cat(outs), torch.cat(sums)


def _exact_attention(s, c, keys_values):
    T, Hq, D = s["q"].shape
    G = Hq // c["Hkv"]
    out = torch.empty(T, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.empty(T, Hq, dtype=torch.float64, device=DEV)
    a = 0
    for b, n in enumerate(s["new"]):
        for g in range(c["Hkv"]):
            k, v = keys_values(b, g)
            at = (slice(a, a + n), slice(g * G, (g + 1) * G))
            out[at], lse[at] = _exact_sequence(s["q"][at].double(), k, v, 1 / math.sqrt(D), c.get("causal", True), c["window"])
        a += n
    return dict(out=out, lse=lse)


def _exact_prompt(s, c):
    at = [0]
    for n in s["new"]:
        at.append(at[-1] + n)
    return _exact_attention(s, c, lambda b, g: tuple(s[x][at[b]:at[b + 1], g].double() for x in "kv"))


def _exact_chunk(s, c):
    def keys_values(b, g):
        pages = s["table"][b, :-(-s["lens"][b] // c["page"])].long()
        return tuple(cache[pages, :, g].reshape(-1, c["D"])[:s["lens"][b]].double() * (1.0 if scale is None else scale[g].double())
                     for cache, scale in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
    return _exact_attention(s, c, keys_values)


def _exact_qknorm(s, c):
    half = c["rot"] // 2

    def made(x, w):
        x = x.double()
        x = x / (x.square().sum(2) / c["D"] + EPS).sqrt()[..., None] * w.double()
        if half:
            row = s["table"][s["pos"].long()].double()
            turn = torch.complex(row[:, :half], row[:, half:])[:, None, :]
            if c["pairs"]:
                z = torch.view_as_complex(x[..., :c["rot"]].reshape(*x.shape[:2], half, 2).contiguous()) * turn
                x[..., :c["rot"]] = torch.view_as_real(z).reshape(*x.shape[:2], c["rot"])
            else:
                z = torch.complex(x[..., :half], x[..., half:c["rot"]]) * turn
                x[..., :half], x[..., half:c["rot"]] = z.real, z.imag
        return x

    q, k = made(s["q"], s["wq"]), made(s["k"], s["wk"])
    caches = []
    for new, cache, scale in ((k, s["kc"], s["ks"]), (s["v"].double(), s["vc"], s["vs"])):
        flat = cache.double().view(-1, c["Hkv"], c["D"])
        if scale is not None:
            new = (new / scale.double()[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
        kept = (s["slots"] >= 0).nonzero()[:, 0]
        flat.index_copy_(0, s["slots"][kept], new[kept])
        caches.append(flat.view(cache.shape))
    return dict(q=q, k=k if c["dense_k"] else None, k_cache=caches[0], v_cache=caches[1])


def _exact_read(s, c):
    def rows(cache, scale):
        x = cache[s["slots"] // c["page"], s["slots"] % c["page"]].double()
        if scale is not None:
            x = x * scale.double()[None, :, None]
        return x.permute(1, 0, 2) if c["by_head"] else x
    return dict(k=rows(s["kc"], s["ks"]), v=rows(s["vc"], s["vs"]) if c["values"] else None)


# -------------------------------------------------------------------------------------------- what a pass cannot avoid
def _pairs(new, lens, causal, window):
    """Visible (token, key) pairs of a sequence."""
    total = 0
    for n, length in zip(new, lens):
        if not causal:
            total += n * length
            continue
        first, last = length - n + 1, length                # keys up to a token's own, of its first and last token
        total += n * (first + last) // 2
        if window:                                          # but the window's
            over = max(0, last - window), max(0, first - 1 - window)
            total -= over[0] * (over[0] + 1) // 2 - over[1] * (over[1] + 1) // 2
    return total


def work(case):
    op, Hkv, D = case["op"], case["Hkv"], case["D"]
    if op in ("prompt", "chunk"):
        T, Hq = case["T"], case["Hq"]
        if op == "prompt":
            new = lens = _split(T, case["B"])
            elem, tables = 2, 0
        else:
            new, lens = _chunks(case)
            elem, tables = (2 if case["kv"] == "bf16" else 1), 4 * sum(-(-n // case["page"]) for n in lens)
        w = case["window"]
        keys = sum(min(length, n + w - 1) if w else length for n, length in zip(new, lens))
        return dict(bytes=4 * T * Hq * D + 4 * T * Hq + 2 * keys * Hkv * D * elem + tables,
                    flops=4 * D * Hq * _pairs(new, lens, case.get("causal", True), w))
    elem = 2 if case["kv"] == "bf16" else 1
    if op == "qknorm":
        T, Hq = case["T"], case["Hq"]
        return dict(bytes=T * (4 * Hq * D + 2 * Hkv * D * (2 + elem) + (2 * Hkv * D if case["dense_k"] else 0) + 4 * case["rot"] + 12) + 4 * D,
                    flops=T * (Hq + Hkv) * (5 * D + 3 * case["rot"]))
    return dict(bytes=case["N"] * (Hkv * D * (elem + 2) * (2 if case["values"] else 1) + 8), flops=case["N"] * Hkv * D * (2 if case["values"] else 1))
