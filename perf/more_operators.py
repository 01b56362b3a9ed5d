"""What stands between the quantised products of a layer: norms with the residual stream
around them, products with bias, activation and residual in their epilogue.  What they are
timed on, their plain forms and their 64-bit references.

Three kinds of case:

  norm    a block's output added to the residual stream and the sum's norm, as fp16 rows
          or as 8-bit codes (returned as the values they stand for)
  linear  a product on 4- or 8-bit codes, or of fp16 rows with 4-bit weights, with bias,
          activation (gated or not) and residual
  mlp     both together: norm into 4-bit codes, gated gate + up product, its quantiser,
          down product onto the residual stream

`own` false computes them in elementary torch operations, in fp32 with one rounding at the
end (norms' sums in fp64); true calls the package.  A case holds its sizes; values come
from the seed.
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6


# ---- cases -------------------------------------------------------------------------------------------------

def _norm(name, M, K, f32=False, add=True, post=False, gate=False, mod=False, center=False, seqs=1, codes=False):
    return dict(name=name, op="norm", M=M, K=K, f32=f32, add=add, post=post, gate=gate, mod=mod, center=center,
                seqs=seqs, codes=codes)


def _linear(name, M, N, K, bits, group=0, bias=False, act="none", glu=False, res="none"):
    return dict(name=name, op="linear", M=M, N=N, K=K, bits=bits, group=group, bias=bias, act=act, glu=glu, res=res)


def _mlp(name, M, K, F):
    return dict(name=name, op="mlp", M=M, K=K, F=F)


def listed():
    return [
        # the next token of one sequence: latency
        _norm("norm_one", 1, 4096),
        # eight prompts of 2048 tokens, fp16 stream
        _norm("norm_prompt", 16384, 4096),
        # eight ragged sequences of a time-conditioned block: the block's output normed too, gates, scales and shifts
        # of each sequence, mean taken off, fp32 stream
        _norm("norm_conditioned", 3000, 3584, f32=True, post=True, gate=True, mod=True, center=True, seqs=8),
        # two prompts straight into the 8-bit codes of the next product, masked and unmasked tokens
        _norm("norm_codes", 4096, 3584, codes=True),
        # one token through the fused query, key and value projection with its bias: latency
        _linear("linear_one", 1, 4608, 3584, 4, bias=True),
        # a ragged serving batch through a square projection onto an fp32 stream
        _linear("linear_o", 1000, 4096, 4096, 4, res="f32"),
        # eight prompts of 2048 tokens through gate and up: the largest
        _linear("linear_glu", 16384, 37888, 3584, 4, act="silu", glu=True),
        # 2048 tokens on 8-bit codes, a plain feed-forward's first half
        _linear("linear_w8", 2048, 12288, 4096, 8, bias=True, act="gelu_tanh"),
        # eight next tokens, weight-only gate and up
        _linear("linear_w4a16", 8, 24576, 4096, 16, group=128, act="silu", glu=True),
        # the same kind of rows down onto the stream, ragged
        _linear("linear_w4a16_down", 13, 4096, 12288, 16, group=64, res="f16"),
        # the feed-forward half of a layer's step: 16 next tokens, and two prompts of 1024
        _mlp("mlp_step", 16, 4096, 12288),
        _mlp("mlp_prompt", 2048, 3584, 18944),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "mlp"])
    if op == "norm":
        codes = rng.random() < 0.4
        K = 64 * _log(rng, 1, 296) if codes else 8 * _log(rng, 4, 2368)
        M = _log(rng, 1, min(16384, 16384 * 4096 // K))
        return dict(op="norm", M=M, K=K, f32=rng.random() < 0.4, add=rng.random() < 0.8, post=rng.random() < 0.4,
                    gate=rng.random() < 0.4, mod=rng.random() < 0.4, center=rng.random() < 0.3,
                    seqs=_log(rng, 1, 32), codes=codes)
    if op == "mlp":
        K, F = 64 * _log(rng, 4, 64), 64 * _log(rng, 4, 296)
        return dict(op="mlp", M=_log(rng, 1, 4096), K=K, F=F)
    bits = rng.choice([4, 4, 8, 16])
    K = 64 * _log(rng, 1, 296)
    M = _log(rng, 1, 32 if bits == 16 else 8192)
    N = 16 * _log(rng, 1, min(2368, 16384 * 37888 * 3584 // 16 // M // K))
    glu = rng.random() < 0.5
    group = rng.choice([g for g in (32, 64, 128, K) if K % g == 0 and (g < 128 or g % 128 == 0)]) if bits == 16 else 0
    return dict(op="linear", M=M, N=N, K=K, bits=bits, group=group, bias=rng.random() < 0.5,
                act=rng.choice(["none", "relu", "relu2", "silu", "silu", "gelu", "gelu_tanh"]), glu=glu,
                res=rng.choice(["none", "f16", "f32"]))


def work(case):
    M, K = case["M"], case["K"]
    if case["op"] == "norm":
        n, stream = M * K, 4 if case["f32"] else 2
        rows = (case["gate"] + 2 * case["mod"]) * case["seqs"] * 2 * K
        return {"bytes": n * stream + (n * (2 + stream) if case["add"] else 0) + (n + 4 * M if case["codes"] else 2 * n)
                + rows + 2 * K, "flops": 10 * n}
    if case["op"] == "mlp":
        F = case["F"]
        return {"bytes": 3 * K * F // 2 + 4 * (2 * F + K) + 4 * M * K, "flops": 6 * M * K * F}
    N, out = case["N"], case["N"] // 2 if case["glu"] else case["N"]
    each = 4 if case["res"] == "f32" else 2
    weights = (N * K + 4 * N if case["bits"] == 8 else N * K // 2
               + (2 * N * (K // case["group"]) if case["bits"] == 16 else 4 * N))
    rows = M * K * case["bits"] // 8 + (0 if case["bits"] == 16 else 4 * M)
    stream = M * out * each * (1 if case["res"] == "none" else 2)
    return {"bytes": weights + rows + (2 * N if case["bias"] else 0) + stream, "flops": 2 * M * N * K}


# ---- inputs ------------------------------------------------------------------------------------------------

def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device=DEVICE) * std


def _codes(gen, bits, *shape):
    """Codes as the quantisers leave them: a bell over most of the range."""
    top = 127 if bits == 8 else 7
    return _normal(gen, *shape, std=top / 2.7).round_().clamp_(-top, top).to(torch.int8)


def _packed(codes):
    """Two 4-bit codes a byte, the even one low."""
    u = codes.view(torch.uint8) & 15
    return u[:, 0::2] | (u[:, 1::2] << 4)


def _fragments(rows):
    """Weight rows (bytes) in the order the package's products read them: 16 rows x 64 bytes a block."""
    N, kb = rows.shape
    groups, steps = -(-N // 16), -(-kb // 64)
    pad = torch.zeros(groups * 16, steps * 64, device=DEVICE, dtype=torch.uint8)
    pad[:N, :kb] = rows
    return pad.view(groups, 16, steps, 4, 16).permute(2, 0, 3, 1, 4).reshape(steps, groups, 1024).contiguous()


def _paired(x):
    """Rows [gates, ups] as blocks of 8 gates and their 8 ups."""
    half = x.shape[0] // 2
    return torch.stack([x[:half].view(half // 8, 8, -1), x[half:].view(half // 8, 8, -1)], 1).reshape(x.shape)


def _weights(gen, N, K, bits, glu):
    codes = _codes(gen, 8 if bits == 8 else 4, N, K)
    rows = codes.view(torch.uint8) if bits == 8 else _packed(codes)
    return codes, _fragments(_paired(rows) if glu else rows)


def _scales(gen, n, typical):
    return (0.5 + torch.rand(n, generator=gen, device=DEVICE)) * typical


def _stream(gen, M, K, f32, far=12.0):
    h = _normal(gen, M, K)
    h[:, 3::97] *= far                                                 # channels that run far out, as streams have
    return h if f32 else h.to(torch.float16)


def _near_one(gen, K):
    return (1.0 + _normal(gen, K, std=0.2)).to(torch.float16)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = {"case": case}
    M, K = case["M"], case["K"]
    if case["op"] == "norm":
        s["h"] = _stream(gen, M, K, case["f32"])
        s["w"] = _near_one(gen, K)
        s["y"] = _normal(gen, M, K, std=0.7).to(torch.float16) if case["add"] else None
        s["wy"] = _near_one(gen, K) if case["add"] and case["post"] else None
        rows = _normal(gen, case["seqs"], 3 * K, std=0.3).to(torch.float16)    # one projection's rows: views of it
        s["gate"] = rows[:, :K] if case["add"] and case["gate"] else None
        s["scale"], s["shift"] = (rows[:, K:2 * K], rows[:, 2 * K:]) if case["mod"] else (None, None)
        s["seq"] = torch.randint(0, case["seqs"], (M,), generator=gen, device=DEVICE).sort()[0].to(torch.int32)
        s["state"] = torch.randint(0, 2, (M,), generator=gen, device=DEVICE).to(torch.uint8)
        return s
    if case["op"] == "mlp":
        F = case["F"]
        s["h"], s["w"] = _stream(gen, M, K, False, far=3.0), _near_one(gen, K)    # a basis has spread them
        s["state"] = torch.randint(0, 2, (M,), generator=gen, device=DEVICE).to(torch.uint8)
        s["up"], s["up_frag"] = _weights(gen, 2 * F, K, 4, True)
        s["up_scale"] = _scales(gen, 2 * F, 0.4 / math.sqrt(K))
        s["down"], s["down_frag"] = _weights(gen, K, F, 4, False)
        s["down_scale"] = _scales(gen, K, 0.4 / math.sqrt(F))
        return s
    N, bits = case["N"], case["bits"]
    s["codes"], s["frag"] = _weights(gen, N, K, bits, case["glu"])
    if bits == 16:
        s["x"] = _normal(gen, M, K).to(torch.float16)
        s["scale"] = (_scales(gen, (K // case["group"]) * N, 0.4 / math.sqrt(K)).view(-1, N)).to(torch.float16)
    else:
        top = 127 if bits == 8 else 7
        a = _codes(gen, bits, M, K)
        s["a"] = a if bits == 8 else _packed(a)
        s["a_scale"] = _scales(gen, M, 2.7 / top)
        s["scale"] = _scales(gen, N, 2.7 / top / math.sqrt(K))
    s["bias"] = _normal(gen, N, std=0.5).to(torch.float16) if case["bias"] else None
    out = N // 2 if case["glu"] else N
    r = _normal(gen, M, out) if case["res"] != "none" else None
    s["r"] = r.to(torch.float16) if case["res"] == "f16" else r
    return s


# ---- plain forms -------------------------------------------------------------------------------------------

def _rate(x, center):
    """Mean and 1 / sqrt(mean square + eps) of rows, in fp64, each rounded once to fp32."""
    x = x.double()
    mean = x.mean(-1, keepdim=True) if center else torch.zeros_like(x[:, :1])
    x = x - mean
    return mean.float(), (1.0 / ((x * x).mean(-1, keepdim=True) + EPS).sqrt()).float()


def _normed(x, w, center):
    mean, rate = _rate(x, center)
    x = x.float()
    if center:
        x = x - mean
    return x * rate * w.float()


def _kept(state, K):
    """Columns that a row keeps: the shared ones and its own state's band (the last two K / 32 are the bands)."""
    band = K // 32
    j = torch.arange(K, device=DEVICE)
    masked = (state != 0)[:, None]
    return (j < K - 2 * band) | (masked & (j < K - band)) | (~masked & (j >= K - band))


def _quantised(x, top):
    """Rows' codes and scales: the divisions in fp64 and rounded once, which is the correctly rounded fp32 division."""
    s = (x.abs().amax(-1, keepdim=True).double() / top).float()
    q = torch.where(s > 0, (x.double() / s.double()).float(), 0.0)
    return q.round().clamp(-top - 1, top), s


def _values(q, scale):
    """What codes stand for, in halves (one pass: the product is rounded as it is written)."""
    return torch.mul(q, scale, out=torch.empty(q.shape, device=DEVICE, dtype=torch.float16))


def _norm_plain(s):
    c = s["case"]
    h, seq = s["h"], s["seq"].long()
    if c["add"]:
        u = _normed(s["y"], s["wy"], c["center"]) if c["post"] else s["y"].float()
        if c["gate"]:
            u = u * s["gate"].float()[seq]
        h = (h.float() + u * 0.5).to(h.dtype)
    n = _normed(h, s["w"], c["center"])
    if c["mod"]:
        n = n * (1.0 + s["scale"].float())[seq] + s["shift"].float()[seq]
    if not c["codes"]:
        return {"x": n.to(torch.float16), "h": h}
    q, scale = _quantised(torch.where(_kept(s["state"], c["K"]), n, 0.0), 127)
    return {"values": _values(q, scale), "h": h}


def _act(t, act):
    if act == "relu":
        return t.clamp(min=0.0)
    if act == "relu2":
        return t.clamp(min=0.0) * t.clamp(min=0.0)
    if act == "silu":
        return t / (1.0 + (-t).exp())
    if act == "gelu":
        return 0.5 * t * torch.erfc(t * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return t / (1.0 + (t * (-2 * math.sqrt(2 / math.pi)) * (1.0 + 0.044715 * t * t)).exp())
    return t


def _gated(t, act, glu):
    if not glu:
        return _act(t, act)
    half = t.shape[1] // 2
    return _act(t[:, :half], act) * t[:, half:]


def _unpacked(a):
    u = torch.stack([a & 15, a >> 4], -1).reshape(a.shape[0], -1).to(torch.int8)
    return torch.where(u > 7, u - 16, u)


def _linear_plain(s):
    c = s["case"]
    w = s["codes"].float()
    if c["bits"] == 16:
        w = w * s["scale"].float().t().repeat_interleave(c["group"], 1)
        t = s["x"].float() @ w.t()
    else:
        a = s["a"] if c["bits"] == 8 else _unpacked(s["a"])
        t = (a.float() @ w.t()) * s["a_scale"][:, None] * s["scale"]
    if c["bias"]:
        t = t + s["bias"].float()
    y = _gated(t, c["act"], c["glu"])
    return y.to(torch.float16) if c["res"] == "none" else (y + s["r"].float()).to(s["r"].dtype)


def _mlp_plain(s):
    K, F = s["case"]["K"], s["case"]["F"]
    n = _normed(s["h"], s["w"], False)
    q, scale = _quantised(torch.where(_kept(s["state"], K), n, 0.0), 7)
    t = (q @ s["up"].float().t()) * scale * s["up_scale"]
    y = _gated(t, "silu", True).to(torch.float16).float()
    q, scale = _quantised(torch.where(_kept(s["state"], F), y, 0.0), 7)
    y = (q @ s["down"].float().t()) * scale * s["down_scale"]
    return (y + s["h"].float()).to(torch.float16)


# ---- the package's calls -----------------------------------------------------------------------------------

def _own(s):
    import paper_2606_04945_amd as sq
    c = s["case"]
    if c["op"] == "norm":
        args = dict(weight=s["w"], post_weight=s["wy"], gate=s["gate"], alpha=0.5, scale=s["scale"], shift=s["shift"],
                    seq=s["seq"], eps=EPS, center=c["center"])
        if not c["codes"]:
            x, h = sq.norm(s["h"], s["y"], **args)
            return {"x": x, "h": h}
        q, scale, h = sq.norm_quant(s["h"], s["y"], state=s["state"], bits=8, **args)
        return {"values": _values(q, scale[:, None]), "h": h}
    if c["op"] == "mlp":
        q, scale, h = sq.norm_quant(s["h"], weight=s["w"], state=s["state"], eps=EPS)
        y = sq.w4a4_linear(q, scale, s["up_frag"], s["up_scale"], act="silu", glu=True)
        q, scale = sq.sgat_quant_act(y, s["state"])
        return sq.w4a4_linear(q, scale, s["down_frag"], s["down_scale"], residual=h)
    args = dict(bias=s["bias"], act=c["act"], glu=c["glu"], residual=s["r"])
    if c["bits"] == 16:
        return sq.w4a16_linear(s["x"], s["frag"], s["scale"], **args)
    f = sq.w8a8_linear if c["bits"] == 8 else sq.w4a4_linear
    return f(s["a"], s["a_scale"], s["frag"], s["scale"], **args)


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    return _norm_plain(s) if op == "norm" else _linear_plain(s) if op == "linear" else _mlp_plain(s)


# ---- 64-bit references -------------------------------------------------------------------------------------

def _unit(x, w, center):
    """Rows of zero mean (if asked) and unit mean square, times w."""
    if center:
        x = x - x.sum(1, keepdim=True) / x.shape[1]
    power = torch.linalg.vector_norm(x, dim=1, keepdim=True).square() / x.shape[1]
    return w.double() * x * torch.rsqrt(power + EPS)


def _visible(x, state):
    x = x.clone()
    K = x.shape[1]
    band = K // 32
    if band:
        x[state == 0, K - 2 * band:K - band] = 0.0
        x[state != 0, K - band:] = 0.0
    return x


def _steps(x, top):
    s = (x.abs().max(1, keepdim=True)[0] / top).float().double()          # scales are held in fp32
    return torch.round((x / torch.where(s == 0, 1.0, s)).float()).double(), s  # ... and so are the quotients


def _activation(t, act):
    if act == "none":
        return t
    if act in ("relu", "relu2"):
        p = torch.relu(t)
        return p if act == "relu" else p ** 2
    if act == "silu":
        return t * torch.sigmoid(t)
    if act == "gelu":
        return t * torch.special.ndtr(t)
    return t * 0.5 * (1 + torch.tanh((2 / math.pi) ** 0.5 * (t + 0.044715 * t ** 3)))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h, pick = s["h"].double(), s["seq"].long()
        if case["add"]:
            u = s["y"].double()
            if case["post"]:
                u = _unit(u, s["wy"], case["center"])
            if case["gate"]:
                u = u * s["gate"].double().index_select(0, pick)
            h = h + u / 2
        n = _unit(h.to(s["h"].dtype).double(), s["w"], case["center"])         # of the stream as it is held
        if case["mod"]:
            n = n + n * s["scale"].double().index_select(0, pick) + s["shift"].double().index_select(0, pick)
        if not case["codes"]:
            return {"x": n, "h": h}
        q, scale = _steps(_visible(n, s["state"]), 127)
        return {"values": q * scale, "h": h}
    if case["op"] == "mlp":
        F = case["F"]
        # codes are defined on fp32 rows: one that lies on another side of a border changes all that follows it
        power = torch.linalg.vector_norm(s["h"].double(), dim=1, keepdim=True).square() / case["K"]
        n = s["h"].float().mul(torch.rsqrt(power + EPS).float()).mul(s["w"].float())
        q, scale = _steps(_visible(n.double(), s["state"]), 7)
        t = torch.matmul(q, s["up"].double().t()) * scale * s["up_scale"].double()
        y = (_activation(t[:, :F], "silu") * t[:, F:]).to(torch.float16).double()      # rows of halves in between
        q, scale = _steps(_visible(y, s["state"]), 7)
        return s["h"].double() + torch.matmul(q, s["down"].double().t()) * scale * s["down_scale"].double()
    N, K, bits = case["N"], case["K"], case["bits"]
    if bits == 16:
        t = torch.zeros(case["M"], N, device=DEVICE, dtype=torch.float64)
        g = case["group"]
        for j in range(K // g):
            t += torch.matmul(s["x"][:, j * g:(j + 1) * g].double(),
                              s["codes"][:, j * g:(j + 1) * g].double().t()) * s["scale"][j].double()
    else:
        a = s["a"].double()
        if bits == 4:
            byte = s["a"].long()
            a = torch.empty(case["M"], K, device=DEVICE, dtype=torch.float64)
            a[:, 0::2] = ((byte & 15) ^ 8) - 8
            a[:, 1::2] = ((byte >> 4) ^ 8) - 8
        t = torch.matmul(a, s["codes"].double().t())
        t *= s["a_scale"].double()[:, None]
        t *= s["scale"].double()
    if case["bias"]:
        t += s["bias"].double()
    half = N // 2
    y = _activation(t[:, :half], case["act"]) * t[:, half:] if case["glu"] else _activation(t, case["act"])
    return y if case["res"] == "none" else y + s["r"].double()
