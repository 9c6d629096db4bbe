"""Cases and plain forms of the serving operators: rmsnorm_quant, gemm_fp8, kv_append, paged_decode.

Where `own` is false, `run` computes an operator with elementary torch operations in 32 bits, rounded once at the end; where it
is true, it calls this library.  `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -100
DEV = "cuda"


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a decode step of 16 sequences: the norm between two layers, launch-bound
        dict(name="norm-16", op="norm", T=16, H=4096, group=128, residual=True),
        # a long prompt (or a batch of them), wide model, scales per 128 columns for the block-scaled product
        dict(name="norm-prompt", op="norm", T=8192, H=8192, group=128, residual=True),
        # quantisation of an odd number of rows with one scale per row, no residual (the input of the first layer)
        dict(name="norm-rows", op="norm", T=1001, H=5120, group=0, residual=False),
        # query/key/value projection of a decode step: 16 rows against a weight matrix, bound by reading the weights
        dict(name="gemm-16", op="gemm", M=16, N=6144, K=4096, out="bf16"),
        # a ragged chunk of a prompt, columns that are no multiple of a tile
        dict(name="gemm-chunk", op="gemm", M=517, N=2624, K=5120, out="bf16"),
        # a whole prompt against a large projection: tensor-core bound
        dict(name="gemm-prompt", op="gemm", M=8192, N=8192, K=8192, out="bf16"),
        # a decode step of 16 sequences
        dict(name="append-16", op="append", T=16, Hq=32, Hkv=8, D=128, rot=128, pairs=False, page=16, kv="bf16", pool=65536),
        # a prompt into an 8-bit cache, partly rotated heads in interleaved pairs
        dict(name="append-prompt", op="append", T=16001, Hq=32, Hkv=8, D=128, rot=64, pairs=True, page=64, kv="e4m3", pool=131072),
        # one sequence, a short history: latency
        dict(name="decode-one", op="decode", B=1, Hq=32, Hkv=8, D=128, page=16, kv="bf16", longest=777, per_head=False, window=0),
        # a serving batch of ragged lengths over 16-token pages
        dict(name="decode-batch", op="decode", B=64, Hq=32, Hkv=8, D=128, page=16, kv="bf16", longest=8192, per_head=False, window=0),
        # few sequences of long context, 8-bit cache, eight query heads to a key-value head
        dict(name="decode-long-e4m3", op="decode", B=4, Hq=64, Hkv=8, D=128, page=64, kv="e4m3", longest=131072, per_head=False, window=0),
        # tokens selected per head (those of the clusters nearest to its query): single-token pages, a table per key-value head
        dict(name="decode-selected", op="decode", B=8, Hq=16, Hkv=16, D=64, page=1, kv="bf16", longest=4096, per_head=True, window=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "gemm", "append", "decode", "decode"])
    if op == "norm":
        H = rng.choice([_log(rng, 64, 16384), 8 * _log(rng, 16, 2048), 128 * _log(rng, 1, 128)])
        return dict(op=op, T=_log(rng, 1, max(1, min(16384, (1 << 26) // H))), H=H, group=rng.choice([0, 128]),
                    residual=rng.random() < 0.7)
    if op == "gemm":
        K = 16 * _log(rng, 8, 768)
        N = rng.choice([_log(rng, 128, 12288), 128 * _log(rng, 1, 96)])
        most = min(8192, (1 << 39) // (N * K))
        return dict(op=op, M=_log(rng, 1, max(1, most)), N=N, K=K, out=rng.choice(["bf16", "bf16", "fp32"]))
    D = rng.choice([64, 96, 128, 128, 256])
    Hkv = rng.choice([1, 2, 4, 8, 16])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 6, 8, 12, 16] if Hkv < 8 else [1, 2, 4, 5, 8])
    kv = rng.choice(["bf16", "e4m3"])
    page = rng.choice([1, 8, 16, 16, 32, 64, 100])
    if op == "append":
        return dict(op=op, T=_log(rng, 1, 16384 * 128 * 8 // (D * max(8, Hkv))), Hq=Hq, Hkv=Hkv, D=D,
                    rot=rng.choice([D, D, D // 2]), pairs=rng.random() < 0.5, page=page, kv=kv, pool=32768)
    B = _log(rng, 1, 64)
    width = Hkv * D * (4 if kv == "bf16" else 2)                      # bytes of one token's keys and values
    tokens = _log(rng, B, max(B, min((1 << 30) // width, 262144)))   # over the whole batch
    per_head = page == 1 and rng.random() < 0.5
    longest = max(1, 2 * tokens // B)
    return dict(op=op, B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, kv=kv, longest=longest, per_head=per_head,
                window=rng.choice([0, 0, 0, max(1, longest // 3)]))


# ------------------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """Cached tokens per sequence (and head): whole-numbered and fixed by the case, spread from about longest / 16 to longest."""
    n = case["B"] * (case["Hkv"] if case["per_head"] else 1)
    L = case["longest"]
    lens = [max(1, L - (i * 5 % n) * (L - L // 16) // n) for i in range(n)]
    return torch.tensor(lens, dtype=torch.int32).view(case["B"], -1)


def _normal(gen, *shape, std=1.0, dtype=torch.bfloat16):
    out = torch.empty(*shape, dtype=dtype, device=DEV)
    return out.normal_(0.0, std, generator=gen)


def _e4m3(gen, *shape, std):
    return _normal(gen, *shape, std=std).to(E4M3)


def _uniform(gen, *shape, lo, hi):
    return torch.empty(*shape, dtype=torch.float32, device=DEV).uniform_(lo, hi, generator=gen)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    if op == "norm":
        T, H = case["T"], case["H"]
        x = _normal(gen, T, H)
        x[:, :: max(1, H // 7)] *= 20.0                     # a few outlier features, as hidden states have
        r = _normal(gen, T, H, std=3.0) if case["residual"] else None
        w = _normal(gen, H, std=0.2) + 1.0
        return dict(x=x, r=r, w=w)
    if op == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        nk, nn = -(-K // 128), -(-N // 128)
        return dict(x=_e4m3(gen, M, K, std=100.0), xs=_uniform(gen, M, nk, lo=0.002, hi=0.02),
                    w=_e4m3(gen, N, K, std=100.0), ws=_uniform(gen, nn, nk, lo=1e-5, hi=4e-4))
    if op == "append":
        T, Hq, Hkv, D, rot, page = (case[k] for k in ("T", "Hq", "Hkv", "D", "rot", "page"))
        pages = -(-case["pool"] // page)
        e = case["kv"] == "e4m3"
        kc, vc = (torch.zeros(pages, page, Hkv, D, dtype=E4M3 if e else torch.bfloat16, device=DEV) for _ in range(2))
        longest = 32768
        freq = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
        angle = torch.arange(longest, device=DEV, dtype=torch.float64)[:, None] * freq[None, :]
        slots = torch.randperm(pages * page, device=DEV, generator=gen)[:T].clone()
        slots[5::97] = -1                                   # padding rows of a batch: nothing is written for them
        # one projection's output holds q, k and v side by side
        qkv = _normal(gen, T, Hq + 2 * Hkv, D)
        return dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], kc=kc, vc=vc, slots=slots,
                    pos=torch.randint(0, longest, (T,), device=DEV, generator=gen, dtype=torch.int32),
                    table=torch.cat([angle.cos(), angle.sin()], 1).float(),
                    ks=_uniform(gen, Hkv, lo=0.005, hi=0.02) if e else None,
                    vs=_uniform(gen, Hkv, lo=0.005, hi=0.02) if e else None)
    B, Hq, Hkv, D, page = (case[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    e = case["kv"] == "e4m3"
    lens = _lengths(case)
    need = -(-lens // page)                                 # pages of each sequence (and head)
    width = int(need.max())
    # tables of one head per sequence share a sequence's tokens; pages are handed out in random order
    pages = int(need.max(1).values.sum()) + 3
    order = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)
    first = torch.cat([torch.zeros(1, dtype=torch.int64), need.max(1).values.long().cumsum(0)[:-1]])
    at = (first[:, None] + torch.arange(width)[None, :]).clamp_(max=pages - 1).to(DEV)
    table = order[at][:, None, :].expand(B, lens.shape[1], width).clone()
    table[torch.arange(width)[None, None, :].to(DEV) >= need.to(DEV)[:, :, None]] = -1
    kc, vc = (_e4m3(gen, pages, page, Hkv, D, std=60.0) if e else _normal(gen, pages, page, Hkv, D) for _ in range(2))
    if not case["per_head"]:
        table, lens = table[:, 0].contiguous(), lens[:, 0].contiguous()
    return dict(q=_normal(gen, B, Hq, D, std=1.5), kc=kc, vc=vc, table=table, lens=lens.to(DEV),
                ks=_uniform(gen, Hkv, lo=0.01, hi=0.025) if e else None,
                vs=_uniform(gen, Hkv, lo=0.01, hi=0.025) if e else None)


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    if own:     # what a serving program keeps between steps: the cache's handle, the workspace, output buffers
        import paper_2608_12629_b200 as cake
        s["cake"] = cake
        op = case["op"]
        if op == "norm":
            T, H, g = case["T"], case["H"], case["group"]
            s["q"] = torch.empty(T, H, dtype=E4M3, device=DEV)
            s["scale"] = torch.empty(T, -(-H // g) if g else 1, dtype=torch.float32, device=DEV)
            s["out_r"] = torch.empty_like(s["x"]) if case["residual"] else None
        elif op == "gemm":
            s["out"] = torch.empty(case["M"], case["N"], dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device=DEV)
            s["buf"] = cake.alloc_gemm_workspace(case["M"], case["N"], case["K"], DEV)
        elif op == "append":
            s["cache"] = cake.PagedCache(s["kc"], s["vc"], s["ks"], s["vs"])
            s["out_q"] = torch.empty(case["T"], case["Hq"], case["D"], dtype=torch.bfloat16, device=DEV)
            s["buf"] = cake.alloc_append_workspace(DEV)
        else:
            s["cache"] = cake.PagedCache(s["kc"], s["vc"], s["ks"], s["vs"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(case["B"], case["Hq"], dtype=torch.float32, device=DEV)
            s["buf"] = cake.alloc_decode_workspace(case["B"], case["Hq"], case["Hkv"], case["D"], DEV)
    return s


# ------------------------------------------------------------------------------------------------------------ passes
def run(s):
    return (_run_own if own else _run_plain)(s, s["case"])


def _run_own(s, c):
    cake, op = s["cake"], c["op"]
    if op == "norm":
        q, scale, _, res = cake.cake_rmsnorm_quant(s["x"], s["w"], s["r"], eps=1e-6, group=c["group"], out_residual=s["out_r"],
                                                   out_q=s["q"], out_scale=s["scale"])
        return dict(q=q, scale=scale, residual=res)
    if op == "gemm":
        return cake.cake_gemm_fp8(s["x"], s["xs"], s["w"], s["ws"], out=s["out"], ws=s["buf"])
    if op == "append":
        q = cake.cake_kv_append(s["cache"], s["k"], s["v"], s["slots"], s["pos"], s["table"], q=s["q"], out_q=s["out_q"],
                                interleaved=c["pairs"], ws=s["buf"])
        return dict(q=q, k_cache=s["kc"], v_cache=s["vc"])
    out, lse = cake.cake_paged_decode(s["q"], s["cache"], s["table"], s["lens"], window=c["window"], out=s["out"],
                                      out_lse=s["lse"], ws=s["buf"])
    return dict(out=out, lse=lse)


def _blocks(scale, rows, cols):
    """Scales of 128-wide blocks spread over the matrix they belong to."""
    for dim, (n, block) in enumerate((rows, cols)):
        if block > 1:
            scale = scale.repeat_interleave(block, dim)[(slice(None),) * dim + (slice(0, n),)]
    return scale


def _run_plain(s, c):
    return globals()["_plain_" + c["op"]](s, c)


def _plain_norm(s, c):
    T, H = c["T"], c["H"]
    x = s["x"].float()
    if s["r"] is not None:
        x = x + s["r"].float()
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) * s["w"].float()
    g = c["group"] or H
    n = -(-H // g)
    padded = torch.zeros(T, n * g, device=DEV)
    padded[:, :H] = y.abs()
    scale = (padded.view(T, n, g).amax(2) / E4M3_MAX).clamp(min=SCALE_MIN)
    q = (y / _blocks(scale, (T, 1), (H, g))).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3)
    return dict(q=q, scale=scale, residual=x.to(torch.bfloat16) if s["r"] is not None else None)


def _plain_gemm(s, c):
    M, N, K = c["M"], c["N"], c["K"]
    x = s["x"].float() * _blocks(s["xs"], (M, 1), (K, 128))
    w = s["w"].float() * _blocks(s["ws"], (N, 128), (K, 128))
    out = x @ w.t()
    return out.to(torch.bfloat16) if c["out"] == "bf16" else out


def _rotate(x, cos, sin, rot, pairs):
    """x [T, heads, D]; cos, sin [T, rot / 2]."""
    x, cos, sin = x.to(cos.dtype), cos[:, None], sin[:, None]
    a, b = (x[..., :rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if pairs else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(s, c):
    cos, sin = s["table"][s["pos"].long()].chunk(2, 1)
    q, k = (_rotate(s[n], cos, sin, c["rot"], c["pairs"]) for n in ("q", "k"))
    v = s["v"].float()
    if s["ks"] is not None:
        k = (k / s["ks"][:, None]).clamp(-E4M3_MAX, E4M3_MAX)
        v = (v / s["vs"][:, None]).clamp(-E4M3_MAX, E4M3_MAX)
    kept = s["slots"] >= 0
    for cache, new in ((s["kc"], k), (s["vc"], v)):
        byte = cache.element_size() == 1
        new = new.to(cache.dtype)
        (cache.view(torch.uint8) if byte else cache).view(-1, c["Hkv"], c["D"])[s["slots"][kept]] = (new.view(torch.uint8) if byte else new)[kept]
    return dict(q=q.to(torch.bfloat16), k_cache=s["kc"], v_cache=s["vc"])


def _plain_decode(s, c):
    B, Hq, Hkv, D, page = (c[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    table = s["table"].clamp(min=0).long()
    lens = s["lens"]
    t = torch.arange(table.shape[-1] * page, device=DEV)
    if c["per_head"]:
        h = torch.arange(Hkv, device=DEV)[None, :, None, None]
        p = torch.arange(page, device=DEV)[None, None, None, :]
        k, v = (cache[table[:, :, :, None], p, h].flatten(2, 3).float() for cache in (s["kc"], s["vc"]))   # [B, Hkv, L, D]
        n = lens[:, :, None, None]
    else:
        k, v = (cache[table].flatten(1, 2).float().transpose(1, 2) for cache in (s["kc"], s["vc"]))
        n = lens[:, None, None, None]
    seen = t < n
    if c["window"]:
        seen = seen & (t >= n - c["window"])
    q = s["q"].float().view(B, Hkv, Hq // Hkv, D) * (1.0 / math.sqrt(D))
    if s["ks"] is not None:
        q = q * s["ks"][None, :, None, None]
    x = (q @ k.transpose(2, 3)).masked_fill(~seen, -math.inf)                  # [B, Hkv, G, L]
    m = x.amax(3, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(3, keepdim=True)
    out = (e / total) @ v
    if s["vs"] is not None:
        out = out * s["vs"][None, :, None, None]
    return dict(out=out.view(B, Hq, D).to(torch.bfloat16), lse=(m + torch.log(total)).view(B, Hq))


# ------------------------------------------------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    return globals()["_exact_" + case["op"]](_inputs(case, seed), case)


def _exact_norm(s, c):
    T, H = c["T"], c["H"]
    x = s["x"].double()
    if s["r"] is not None:
        x += s["r"].double()
    norm = (x.square().sum(1) / H + 1e-6).sqrt()
    y = x / norm[:, None] * s["w"].double()
    g = c["group"] or H
    q, scales = torch.empty_like(y), []
    for a in range(0, H, g):
        part = y[:, a:a + g]
        sc = torch.clamp(part.abs().max(1).values / E4M3_MAX, min=SCALE_MIN)
        q[:, a:a + g] = part / sc[:, None]
        scales.append(sc)
    return dict(q=q, scale=torch.stack(scales, 1), residual=x if s["r"] is not None else None)


def _exact_gemm(s, c):
    out = torch.zeros(c["M"], c["N"], dtype=torch.float64, device=DEV)
    col = torch.arange(c["N"], device=DEV) // 128
    for kb in range(s["xs"].shape[1]):
        a, b = (s[n][:, 128 * kb:128 * kb + 128].double() for n in ("x", "w"))
        out += (a @ b.t()) * s["xs"][:, kb].double()[:, None] * s["ws"][:, kb].double()[col][None, :]
    return out


def _exact_append(s, c):
    half = c["rot"] // 2
    row = s["table"][s["pos"].long()].double()
    turn = torch.complex(row[:, :half], row[:, half:])[:, None, :]

    def rotated(x):
        x = x.double().clone()
        if c["pairs"]:
            z = torch.view_as_complex(x[..., :c["rot"]].reshape(*x.shape[:2], half, 2).contiguous()) * turn
            x[..., :c["rot"]] = torch.view_as_real(z).reshape(*x.shape[:2], c["rot"])
        else:
            z = torch.complex(x[..., :half], x[..., half:c["rot"]]) * turn
            x[..., :half], x[..., half:c["rot"]] = z.real, z.imag
        return x

    caches = []
    for new, cache, scale in ((rotated(s["k"]), s["kc"], s["ks"]), (s["v"].double(), s["vc"], s["vs"])):
        flat = cache.double().view(-1, c["Hkv"], c["D"])
        if scale is not None:
            new = (new / scale.double()[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
        kept = (s["slots"] >= 0).nonzero()[:, 0]
        flat.index_copy_(0, s["slots"][kept], new[kept])
        caches.append(flat.view(cache.shape))
    return dict(q=rotated(s["q"]), k_cache=caches[0], v_cache=caches[1])


def _exact_decode(s, c):
    B, Hq, Hkv, D, page = (c[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    out = torch.zeros(B, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.empty(B, Hq, dtype=torch.float64, device=DEV)
    lens = s["lens"].cpu()
    for b in range(B):
        for h in range(Hkv):
            n = int(lens[b, h] if c["per_head"] else lens[b])
            pages = (s["table"][b, h] if c["per_head"] else s["table"][b])[:-(-n // page)].long()
            a = max(0, n - c["window"]) if c["window"] else 0
            k, v = (cache[pages, :, h].reshape(-1, D)[a:n].double() for cache in (s["kc"], s["vc"]))
            x = s["q"][b, h * G:(h + 1) * G].double() @ k.t() / math.sqrt(D)
            if s["ks"] is not None:
                x = x * s["ks"][h].double()
                v = v * s["vs"][h].double()
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(x, 1)
            out[b, h * G:(h + 1) * G] = torch.softmax(x, 1) @ v
    return dict(out=out, lse=lse)


# -------------------------------------------------------------------------------------------- what a pass cannot avoid
def work(case):
    op = case["op"]
    if op == "norm":
        T, H, g = case["T"], case["H"], case["group"]
        scales = 4 * T * (-(-H // g) if g else 1)
        return dict(bytes=T * H * ((2 + 2 + 2 + 1) if case["residual"] else (2 + 1)) + 2 * H + scales, flops=8 * T * H)
    if op == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        nk, nn = -(-K // 128), -(-N // 128)
        return dict(bytes=M * K + N * K + 4 * (M + nn) * nk + M * N * (2 if case["out"] == "bf16" else 4), flops=2 * M * N * K)
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    elem = 2 if case["kv"] == "bf16" else 1
    if op == "append":
        T = case["T"]
        return dict(bytes=T * (4 * Hq * D + 2 * Hkv * D * (2 + elem) + 4 * case["rot"] + 12), flops=T * (Hq + Hkv) * case["rot"] * 3)
    lens = _lengths(case).long()
    if case["window"]:
        lens = lens.clamp(max=case["window"])
    tokens = int(lens.sum()) * (1 if case["per_head"] else Hkv)
    entries = int((-(-lens // case["page"])).sum())
    return dict(bytes=tokens * D * 2 * elem + 4 * case["B"] * Hq * D + 4 * entries + 4 * case["B"] * Hq,
                flops=4 * tokens * (Hq // Hkv) * D)
