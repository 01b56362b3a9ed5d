"""The attention side of a quantised layer's step, and its weight-only products:
what they are timed on, their plain forms and their 64-bit references.

Four kinds of case:

  rope    rotary positions on a strided view of a fused projection's output
  append  rotation of q and k, keys and values into the paged 8-bit cache, and
          the pages written read back as the values they stand for
  attn    attention over the paged 8-bit cache (one scale per page and head)
  w4      few rows times 4-bit weights with one scale per group of inputs

`own` false computes them in elementary torch operations, in fp32 with one
rounding at the end; true calls the package.  A case holds its sizes; ragged
lengths come from its number `mix` alone, values from the seed.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"


# ---- cases -------------------------------------------------------------------------------------------------

def _rope(name, T, H, D, rot, pairs, scaling, far, transpose):
    return dict(name=name, op="rope", T=T, H=H, D=D, rot=rot, pairs=pairs, scaling=scaling, far=far,
                transpose=transpose)


def _append(name, B, Hq, Hkv, D, page, new, old, rot, pairs, mix):
    return dict(name=name, op="append", B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, new=new, old=old, rot=rot, pairs=pairs,
                mix=mix)


def _attn(name, B, Hq, Hkv, D, page, new, old, causal, window, lse, mix):
    return dict(name=name, op="attn", B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, new=new, old=old, causal=causal,
                window=window, lse=lse, mix=mix)


def _w4(name, M, N, K, group):
    return dict(name=name, op="w4", M=M, N=N, K=K, group=group)


def listed():
    return [
        # the queries of 16 sequences' next tokens (32 heads of 128): latency
        _rope("rope_step", 16, 32, 128, 128, False, "none", 4096, False),
        # 8 x 2048 tokens of 28 heads far into a context stretched eight times
        _rope("rope_prompt", 16384, 28, 128, 128, False, "yarn", 262144, False),
        # one new token for each of 16 sequences, as many key as query heads
        _append("append_step", 16, 32, 32, 128, 16, 1, 4096, 128, False, 1),
        # prompts of up to 2048 tokens, 28 query heads on 4 key heads
        _append("append_prompt", 8, 28, 4, 128, 64, 2048, 100, 128, False, 2),
        # one sequence's next token over a short cache: latency
        _attn("attn_step_one", 1, 32, 32, 128, 64, 1, 517, True, 0, False, 3),
        # the next tokens of 32 sequences of mixed lengths
        _attn("attn_step_batch", 32, 28, 4, 128, 64, 1, 8192, True, 0, True, 4),
        # two sequences with very long caches, 8 query heads to a key head
        _attn("attn_step_long", 2, 64, 8, 128, 128, 1, 131072, True, 0, False, 5),
        # a block of 32 tokens denoised together, seeing the prompt and each other
        _attn("attn_block", 8, 32, 32, 128, 32, 32, 2048, False, 0, False, 6),
        # 8 prompts of up to 2048 tokens, every token seeing every other
        _attn("attn_prompt", 8, 28, 4, 128, 64, 2048, 0, False, 0, True, 7),
        # the next 512 tokens of two long prompts, each token seeing those before it
        _attn("attn_chunk", 2, 28, 4, 128, 64, 512, 8192, True, 0, False, 8),
        # one token through a square projection: latency
        _w4("w4_one", 1, 4096, 4096, 128),
        # 16 tokens through the fused gate and up projection, finer groups
        _w4("w4_rows", 16, 37888, 3584, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attn", "attn", "w4"])
    D = rng.choice([64, 80, 96, 128, 128, 128])
    if kind == "rope":
        H = rng.choice([4, 8, 28, 32])
        T = min(_log(rng, 1, 16384), 16384 * 28 // H // max(1, D // 64))
        rot = rng.choice([D, D, D // 2 // 16 * 16])
        return dict(op="rope", T=T, H=H, D=D, rot=rot, pairs=rng.random() < 0.4,
                    scaling=rng.choice(["none", "linear", "ntk", "yarn"]), far=_log(rng, 64, 1 << 20),
                    transpose=rng.random() < 0.25)
    Hkv, G = rng.choice([(32, 1), (8, 4), (4, 7), (8, 8), (2, 5)])
    page = rng.choice([16, 32, 64, 128])
    mix = rng.randrange(1 << 20)
    if kind == "append":
        B = _log(rng, 1, 64)
        new = min(_log(rng, 1, 2048), max(1, 8192 // B))
        return dict(op="append", B=B, Hq=Hkv * G, Hkv=Hkv, D=D, page=page, new=new, old=_log(rng, 1, 4096), rot=D,
                    pairs=rng.random() < 0.4, mix=mix)
    if kind == "attn":
        B = _log(rng, 1, 64)
        causal = rng.random() < 0.6
        window = _log(rng, 16, 4096) if rng.random() < 0.2 else 0
        if rng.random() < 0.5:                         # next tokens
            new, old = 1, _log(rng, 1, min(131072, (7 << 18) // (B * Hkv)))
        else:                                          # blocks and prompts
            new = _log(rng, 2, 2048)
            B = max(1, min(B, 12288 * 28 // (new * Hkv * G)))
            old = _log(rng, 1, max(2, min(16384, (1 << 28) // (B * new * Hkv * G))))
        return dict(op="attn", B=B, Hq=Hkv * G, Hkv=Hkv, D=D, page=page, new=new, old=old, causal=causal,
                    window=window, lse=rng.random() < 0.3, mix=mix)
    K = 64 * _log(rng, 4, 296)
    group = rng.choice([g for g in (32, 64, 128, K) if K % g == 0 and (g < 128 or g % 128 == 0)])
    N = 8 * _log(rng, 8, min(4736, 37888 * 3584 // 8 // K))
    return dict(op="w4", M=_log(rng, 1, 32), N=N, K=K, group=group)


def _lengths(case):
    """(new tokens, total length) of each sequence: ragged, the first one the longest."""
    r = random.Random(case["mix"])
    new, total = [], []
    for b in range(case["B"]):
        n = case["new"] if b == 0 or case["new"] == 1 else r.randint(max(1, case["new"] // 2), case["new"])
        o = case["old"] if b == 0 else r.randint(case["old"] // 2, case["old"])
        new.append(n)
        total.append(n + o)
    return new, total


def _visible(case):
    """Sum over query tokens of the keys each one sees, and over sequences of the keys any of them sees."""
    pairs = keys = 0
    w = case["window"]
    for n, L in zip(*_lengths(case)):
        first = max(0, L - n - w + 1) if w else 0
        keys += L - first
        for p in range(L - n, L):
            hi = p + 1 if case["causal"] else L
            pairs += hi - (max(0, p - w + 1) if w else 0)
    return pairs, keys


def work(case):
    if case["op"] == "rope":
        n = case["T"] * case["H"] * case["D"]
        return {"bytes": 4 * n + 4 * case["T"] + 4 * case["rot"], "flops": 3 * n * case["rot"] / case["D"]}
    if case["op"] == "append":
        new, total = _lengths(case)
        T, D, page = sum(new), case["D"], case["page"]
        touched = sum((L - 1) // page - (L - n) // page + 1 for n, L in zip(new, total))
        values = touched * page * case["Hkv"] * D * 2
        return {"bytes": 4 * T * case["Hkv"] * D + 2 * T * case["Hkv"] * D + 4 * T * case["Hq"] * D + 3 * values,
                "flops": 3 * T * (case["Hq"] + case["Hkv"]) * case["rot"] + 4 * T * case["Hkv"] * D + values}
    if case["op"] == "attn":
        pairs, keys = _visible(case)
        T = sum(_lengths(case)[0])
        return {"bytes": 2 * keys * case["Hkv"] * case["D"] + 8 * keys // case["page"] * case["Hkv"]
                + 4 * T * case["Hq"] * case["D"] + (4 * T * case["Hq"] if case["lse"] else 0),
                "flops": 4 * case["D"] * case["Hq"] * pairs}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": N * K // 2 + 2 * N * (K // case["group"]) + 2 * M * K + 2 * M * N, "flops": 2 * M * N * K}


# ---- inputs ------------------------------------------------------------------------------------------------

def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device=DEVICE) * std


def _frequencies(rot, scaling):
    """Radians per position of each pair (fp64) and the amplitude of the rotation, base 1e6, stretched 8 times."""
    base, factor, orig = 1e6, 8.0, 32768.0
    j = torch.arange(rot // 2, device=DEVICE, dtype=torch.float64)
    if scaling == "ntk" and rot > 2:
        base *= factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * j / rot)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":
        turns = orig * f / (2 * math.pi)               # turns over the original context: 32 and more stay, 1 and
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)  # fewer are stretched
        return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _table(case, gen, total):
    """A page table of shuffled pages with a few unused ones, and the number of pages."""
    per = [-(-L // case["page"]) for L in total]
    pages = sum(per) + 3
    order = torch.randperm(pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.full((case["B"], max(per)), -1, device=DEVICE, dtype=torch.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def _cache(case, gen, pages):
    """Codes and scales of normal keys and values, some key channels several times as large."""
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    k = _normal(gen, pages, Hkv, page, D, std=26.0)
    k[..., 3::37] *= 1.7
    v = _normal(gen, pages, Hkv, D, page, std=33.0)
    scale = lambda: (0.6 + 0.8 * torch.rand(pages, Hkv, generator=gen, device=DEVICE)) * 0.03  # noqa: E731
    return {"k": k.round_().clamp_(-127, 127).to(torch.int8), "v": v.round_().clamp_(-127, 127).to(torch.int8),
            "k_scale": scale(), "v_scale": scale()}


def _ints(v):
    return torch.tensor(v, device=DEVICE, dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "rope":
        T, H, D = case["T"], case["H"], case["D"]
        fused = _normal(gen, T, (H + 2) * D).to(torch.float16)            # a projection's output rows
        s["x"] = fused[:, :H * D].view(T, H, D)
        s["pos"] = torch.randint(0, case["far"], (T,), generator=gen, device=DEVICE, dtype=torch.int32)
        s["freq"], s["amp"] = _frequencies(case["rot"], case["scaling"])
        return s
    if case["op"] == "w4":
        M, N, K, g = case["M"], case["N"], case["K"], case["group"]
        s["x"] = _normal(gen, M, K).to(torch.float16)
        codes = _normal(gen, N, K, std=2.6).round_().clamp_(-7, 7).to(torch.int8).view(torch.uint8) & 15
        s["w"] = codes[:, 0::2] | (codes[:, 1::2] << 4)                   # two codes a byte, the even one low
        s["scale"] = ((0.5 + torch.rand(K // g, N, generator=gen, device=DEVICE)) * 0.007).to(torch.float16)
        # the same bytes in the order the package's products read them: 16 rows x 64 bytes a block
        rows, steps = -(-N // 16), -(-K // 128)
        pad = torch.zeros(rows * 16, steps * 64, device=DEVICE, dtype=torch.uint8)
        pad[:N, :K // 2] = s["w"]
        s["frag"] = pad.view(rows, 16, steps, 4, 16).permute(2, 0, 3, 1, 4).reshape(steps, rows, 1024).contiguous()
        return s
    new, total = _lengths(case)
    T, Hq, Hkv, D, page = sum(new), case["Hq"], case["Hkv"], case["D"], case["page"]
    s["table"], pages = _table(case, gen, total)
    s.update(_cache(case, gen, pages))
    s["cu"] = _ints([sum(new[:b]) for b in range(case["B"] + 1)])
    s["lens"] = _ints(total)
    if case["op"] == "append":
        fused = _normal(gen, T, (Hq + 2 * Hkv) * D)
        fused[:, Hq * D + 3:(Hq + Hkv) * D:37] *= 3.0
        fused = fused.to(torch.float16)
        s["q"] = fused[:, :Hq * D].view(T, Hq, D)
        s["knew"] = fused[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
        s["vnew"] = fused[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        s["freq"], s["amp"] = _frequencies(case["rot"], "none")
        s["touched"] = torch.cat([s["table"][b, (L - n) // page:(L - 1) // page + 1]
                                  for b, (n, L) in enumerate(zip(new, total))])
    else:
        s["q"] = _normal(gen, T, Hq, D).to(torch.float16)
        s["most"] = max(new)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------

def _rotate(x, pos, freq, amp, rot, pairs, transpose=False):
    """fp32 rotation of the first `rot` entries of [T, H, D]; the angles, of far positions, in fp64."""
    a = pos.double()[:, None, None] * freq
    c, sn = (a.cos() * amp).float(), (a.sin() * (-amp if transpose else amp)).float()
    x = x.float()
    if pairs:
        u, v = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        u, v = x[..., :rot // 2], x[..., rot // 2:rot]
    y = x.clone()
    if pairs:
        y[..., 0:rot:2], y[..., 1:rot:2] = u * c - v * sn, v * c + u * sn
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u * c - v * sn, v * c + u * sn
    return y


def _rope_plain(s):
    c = s["case"]
    return _rotate(s["x"], s["pos"], s["freq"], s["amp"], c["rot"], c["pairs"], c["transpose"]).to(torch.float16)


def _tokens(s, T):
    """Sequence, index in it and cache position of each token."""
    t = torch.arange(T, device=DEVICE)
    cu = s["cu"].long()
    b = torch.searchsorted(cu, t, right=True) - 1
    i = t - cu[b]
    return b, i, s["lens"].long()[b] - (cu[b + 1] - cu[b]) + i


def _append_plain(s):
    c = s["case"]
    D, page, T = c["D"], c["page"], s["q"].shape[0]
    b, i, pos = _tokens(s, T)
    touched = s["touched"].long()
    at = torch.zeros(s["k"].shape[0], device=DEVICE, dtype=torch.long)
    at[touched] = torch.arange(len(touched), device=DEVICE)
    blk, slot = at[s["table"].long()[b, pos // page]], pos % page
    first = torch.full((len(touched),), page, device=DEVICE).index_reduce_(0, blk, slot, "amin")
    kept = torch.arange(page, device=DEVICE) < first[:, None]             # [block, slot]: already there
    q = _rotate(s["q"], pos, s["freq"], s["amp"], c["rot"], c["pairs"]).to(torch.float16)
    out = {"q": q}
    k = _rotate(s["knew"], pos, s["freq"], s["amp"], c["rot"], c["pairs"])
    for name, x in (("k", k), ("v", s["vnew"].float())):
        codes = s[name][touched].float()
        if name == "v":
            codes = codes.transpose(2, 3)                                 # [block, head, slot, D]
        old = s[name + "_scale"][touched]
        most = torch.zeros_like(old).index_reduce_(0, blk, x.abs().amax(-1), "amax")
        new = torch.maximum(torch.where(first[:, None] > 0, old, 0.0), most / 127)
        ratio = torch.where(new > old, old / new, 1.0)[:, :, None, None]
        codes = torch.where(kept[:, None, :, None], (codes * ratio).round(), codes)
        codes[blk, :, slot] = (x / new[blk][..., None]).nan_to_num(0.0).round().clamp(-128, 127)
        out[name] = (codes * new[:, :, None, None]).to(torch.float16)
    return out


def _gathered(s, dtype):
    """Keys and values of every sequence [B, Hkv, L, D] as the values they stand for."""
    pages = s["table"].long().clamp(min=0)
    k = s["k"][pages].to(dtype) * s["k_scale"][pages].to(dtype)[..., None, None]      # [B, pages, Hkv, page, D]
    v = s["v"][pages].to(dtype) * s["v_scale"][pages].to(dtype)[..., None, None]
    B, n, H, page, D = k.shape
    return (k.permute(0, 2, 1, 3, 4).reshape(B, H, n * page, D),
            v.permute(0, 2, 1, 4, 3).reshape(B, H, n * page, D))


def _attn_plain(s):
    c = s["case"]
    T, Hq, D = s["q"].shape
    Hkv, most = c["Hkv"], s["most"]
    G = Hq // Hkv
    b, i, _ = _tokens(s, T)
    k, v = _gathered(s, torch.float32)
    q = torch.zeros(c["B"], most, Hq, D, device=DEVICE)
    q[b, i] = s["q"].float()
    q = q.view(c["B"], most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(c["B"], Hkv, most * G, D)
    x = (q @ k.transpose(2, 3).contiguous()) / math.sqrt(D)
    lens, cu = s["lens"].long(), s["cu"].long()
    at = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + torch.arange(most, device=DEVICE)      # [B, query] position
    key = torch.arange(x.shape[3], device=DEVICE)
    seen = (key < lens[:, None])[:, None].expand(-1, most, -1)
    if c["causal"]:
        seen = seen & (key <= at[..., None])
    if c["window"]:
        seen = seen & (key > at[..., None] - c["window"])
    x.masked_fill_(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x = (x - m).exp_()
    total = x.sum(-1, keepdim=True)
    y = (x @ v) / torch.where(total == 0, 1.0, total)
    y = y.view(c["B"], Hkv, most, G, D).permute(0, 2, 1, 3, 4).reshape(c["B"], most, Hq, D)[b, i].to(torch.float16)
    if not c["lse"]:
        return y
    lse = (m + total.log()).view(c["B"], Hkv, most, G).permute(0, 2, 1, 3).reshape(c["B"], most, Hq)[b, i]
    return {"out": y, "lse": lse}


def _w4_plain(s):
    lo, hi = s["w"] & 15, s["w"] >> 4
    w = torch.stack([lo, hi], -1).reshape(s["w"].shape[0], -1).to(torch.int8)
    w = torch.where(w > 7, w - 16, w).float()
    w = w * s["scale"].float().t().repeat_interleave(s["case"]["group"], 1)
    return (s["x"].float() @ w.t()).to(torch.float16)


# ---- the package's calls -----------------------------------------------------------------------------------

def _own(s):
    import paper_2606_04945_amd as sq
    c = s["case"]
    layout = "pairs" if c.get("pairs") else "half"
    if c["op"] == "rope":
        return sq.rope(s["x"], s["freq"], s["pos"], layout=layout, amplitude=s["amp"], transpose=c["transpose"])
    if c["op"] == "w4":
        return sq.w4a16_gemm_frag(s["x"], s["frag"], s["scale"])
    cache = sq.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if c["op"] == "append":
        q = sq.kv_append(cache, s["knew"], s["vnew"], s["cu"], s["lens"], s["table"], freq=s["freq"], q=s["q"],
                         layout=layout, amplitude=s["amp"])
        k, v = sq.kv_read(cache, s["touched"])
        return {"q": q, "k": k, "v": v}
    r = sq.attn_kv8(s["q"], cache, s["cu"], s["lens"], s["table"], causal=c["causal"], window=c["window"],
                    want_lse=c["lse"])
    return {"out": r[0], "lse": r[1]} if c["lse"] else r


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    if op == "rope":
        return _rope_plain(s)
    if op == "append":
        return _append_plain(s)
    return _attn_plain(s) if op == "attn" else _w4_plain(s)


# ---- 64-bit references -------------------------------------------------------------------------------------

def _turned(x, pos, freq, amp, rot, pairs, transpose=False):
    """The rotation as a product of complex numbers, in fp64."""
    x = x.double()
    head = x[..., :rot]
    z = (torch.complex(head[..., 0::2].contiguous(), head[..., 1::2].contiguous()) if pairs else
         torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()))
    a = pos.double()[:, None] * freq[None]
    z = z * torch.polar(torch.full_like(a, amp), -a if transpose else a)[:, None]
    y = torch.stack([z.real, z.imag], -1).flatten(-2) if pairs else torch.cat([z.real, z.imag], -1)
    return torch.cat([y, x[..., rot:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _turned(s["x"], s["pos"], s["freq"], s["amp"], case["rot"], case["pairs"], case["transpose"])
    if case["op"] == "w4":
        N, K, g = case["N"], case["K"], case["group"]
        byte = s["w"].long()
        w = torch.empty(N, K, device=DEVICE, dtype=torch.float64)
        w[:, 0::2] = ((byte & 15) ^ 8) - 8
        w[:, 1::2] = ((byte >> 4) ^ 8) - 8
        y = torch.zeros(case["M"], N, device=DEVICE, dtype=torch.float64)
        for j in range(K // g):
            y += (s["x"][:, j * g:(j + 1) * g].double() @ w[:, j * g:(j + 1) * g].t()) * s["scale"][j].double()
        return y
    new, total = _lengths(case)
    D, page, Hkv, G = case["D"], case["page"], case["Hkv"], case["Hq"] // case["Hkv"]
    if case["op"] == "append":
        pos = torch.cat([torch.arange(L - n, L, device=DEVICE) for n, L in zip(new, total)])
        turn = lambda x: _turned(x, pos, s["freq"], s["amp"], case["rot"], case["pairs"])  # noqa: E731
        rows = {"k": turn(s["knew"]), "v": s["vnew"].double()}
        out = {"q": turn(s["q"]), "k": [], "v": []}
        t = 0
        for b, (n, L) in enumerate(zip(new, total)):
            p = L - n
            while p < L:                                # the part of each page that this sequence writes
                lo, end = p % page, min(L, (p // page + 1) * page)
                at = int(s["table"][b, p // page])
                for name in ("k", "v"):
                    x = rows[name][t:t + end - p].permute(1, 0, 2)                    # [Hkv, tokens, D]
                    had = s[name][at].double()
                    had = had.transpose(1, 2).clone() if name == "v" else had.clone()
                    scale = x.abs().amax((1, 2)) / 127
                    if lo:
                        was = s[name + "_scale"][at].double()
                        scale = torch.maximum(scale, was)
                        had[:, :lo] = (had[:, :lo] * (was / scale)[:, None, None]).round()
                    had[:, lo:lo + end - p] = (x / scale[:, None, None]).round()
                    out[name].append(had * scale[:, None, None])
                t, p = t + end - p, end
        return {"q": out["q"], "k": torch.stack(out["k"]), "v": torch.stack(out["v"])}
    outs, lses, t = [], [], 0
    for b, (n, L) in enumerate(zip(new, total)):
        own_pages = s["table"][b, :-(-L // page)].long()
        kc = s["k"][own_pages].double() * s["k_scale"][own_pages].double()[..., None, None]
        vc = s["v"][own_pages].double() * s["v_scale"][own_pages].double()[..., None, None]
        k = kc.transpose(0, 1).reshape(Hkv, -1, D)[:, :L]
        v = vc.permute(1, 0, 3, 2).reshape(Hkv, -1, D)[:, :L]
        q = s["q"][t:t + n].double().view(n, Hkv, G, D)
        p, j = torch.arange(L - n, L, device=DEVICE)[:, None], torch.arange(L, device=DEVICE)[None]
        hidden = torch.zeros(n, L, device=DEVICE, dtype=torch.bool)
        if case["causal"]:
            hidden |= j > p
        if case["window"]:
            hidden |= j <= p - case["window"]
        ys, zs = [], []
        for h in range(Hkv):
            x = torch.matmul(q[:, h].reshape(n * G, D), k[h].t()).view(n, G, L) * D ** -0.5
            x.masked_fill_(hidden[:, None], -math.inf)
            z = torch.logsumexp(x, -1)
            ys.append(torch.matmul((x - z[..., None]).exp().view(n * G, L), v[h]).view(n, G, D))
            zs.append(z)
        outs.append(torch.stack(ys, 1).reshape(n, Hkv * G, D))
        lses.append(torch.stack(zs, 1).reshape(n, Hkv * G))
        t += n
    y = torch.cat(outs)
    return {"out": y, "lse": torch.cat(lses)} if case["lse"] else y
