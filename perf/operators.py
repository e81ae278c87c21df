"""Operators around a target model's attention cache and its next token, and what one pass through each has to return:

  append   norms of queries and keys for each head (or none), position rotation and the append to the cache in one pass; the cache
           holds fp16, or 8 bits per value: int8 or e4m3 codes with one fp16 scale per cached row and head
  read     rows of an 8-bit cache back as fp16
  attn     attention of a verification pass (committed prefix, then draft keys behind a tree mask) over an 8-bit cache
  sample   next tokens from given uniform numbers, with temperature, top-k, top-p and min-p

Without `own` a pass is elementary torch operations in 32 bits (64 for the sampling weights, whose borders decide a token).
Definitions shared by all of them:
  int8 cache   s = amax / 127 rounded up to four significant bits (a multiple of 2^-24, at most 512), code = round(v / s) within +-127
  e4m3 cache   s = amax / 448 rounded up to a power of two (at least 2^-15), code = e4m3(v / s), kept below the end of fp16
  A code times its scale is an fp16 number, so reading back rounds nothing."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
D_ATTN = 128     # head dimension of the attention
HEADS = [(32, 8), (64, 8), (40, 8), (16, 2), (12, 2), (8, 8), (28, 4)]
MOST_SCORES = 60 * 64 * 16061      # query rows x keys of the largest attention
MOST_ROWS = 131072                 # rows of the longest cache


def listed():
    return [
        # plain decoding: one token of an 8B-sized layer with head norms, fp16 cache; latency is all there is
        {"name": "append_fp16_m1", "kind": "append", "fmt": "fp16", "norm": True, "M": 1, "P": 2048, "Hq": 32, "Hkv": 8, "D": 128},
        # tree verification of 60 nodes, 70B heads, int8 cache
        {"name": "append_int8_m60", "kind": "append", "fmt": "int8", "norm": True, "M": 60, "P": 8191, "Hq": 64, "Hkv": 8, "D": 128},
        # a prompt's chunk written to an e4m3 cache, no norms
        {"name": "append_e4m3_m4096", "kind": "append", "fmt": "e4m3", "norm": False, "M": 4096, "P": 1000, "Hq": 32, "Hkv": 8, "D": 128},
        # a short stretch of a cache handed to a consumer that wants fp16, four heads
        {"name": "read_int8_777", "kind": "read", "fmt": "int8", "rows": 777, "first": 130, "Hkv": 4, "D": 128},
        # a whole long cache read back
        {"name": "read_e4m3_65536", "kind": "read", "fmt": "e4m3", "rows": 65536, "first": 3, "Hkv": 8, "D": 128},
        # plain decoding behind a prompt of ordinary length, 70B heads
        {"name": "attn_int8_m1_p2048", "kind": "attn", "fmt": "int8", "M": 1, "P": 2048, "Hq": 64, "Hkv": 8, "pad": 0},
        # sequence verification (draft of 6) behind the longest context
        {"name": "attn_e4m3_m7_p131065", "kind": "attn", "fmt": "e4m3", "M": 7, "P": 131065, "Hq": 32, "Hkv": 8, "pad": 0},
        # tree verification of 60 nodes behind a long document, 70B heads: the most arithmetic
        {"name": "attn_int8_m60_p16001", "kind": "attn", "fmt": "int8", "M": 60, "P": 16001, "Hq": 64, "Hkv": 8, "pad": 0},
        # a tree padded to a fixed size (its last rows see nothing), ragged prefix, heads in groups of seven
        {"name": "attn_e4m3_m37_p3333_pad", "kind": "attn", "fmt": "e4m3", "M": 37, "P": 3333, "Hq": 28, "Hkv": 4, "pad": 5},
        # one token of a small vocabulary, top-k as chat programs set it
        {"name": "sample_m1_v32000_k", "kind": "sample", "M": 1, "V": 32000, "filters": "k", "banned": False},
        # one token of a large vocabulary, nucleus only: no candidate list bounds the work
        {"name": "sample_m7_v128256_p", "kind": "sample", "M": 7, "V": 128256, "filters": "p", "banned": False},
        # a token for every node of a verified tree, all filters, tokens banned by a grammar
        {"name": "sample_m60_v128256_all", "kind": "sample", "M": 60, "V": 128256, "filters": "all", "banned": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "read", "attn", "attn", "attn", "sample", "sample"])
    fmt = rng.choice(["int8", "e4m3"])
    Hq, Hkv = rng.choice(HEADS)
    if kind == "append":
        M = _log_int(rng, 1, 4096)
        cache = rng.choice(["fp16", "int8", "e4m3"])   # without norms an fp16 cache takes rope_append, which is measured elsewhere
        return {"kind": kind, "fmt": cache, "norm": cache == "fp16" or rng.random() < 0.7, "M": M, "P": _log_int(rng, 1, 20000),
                "Hq": Hq, "Hkv": Hkv, "D": rng.choice([64, 80, 112, 128, 128, 256]) if M * Hq < 65536 else 128}
    if kind == "read":
        return {"kind": kind, "fmt": fmt, "rows": _log_int(rng, 1, 65536), "first": rng.randint(0, 999), "Hkv": Hkv, "D": 128}
    if kind == "attn":
        M = _log_int(rng, 1, 64) if rng.random() < 0.6 else rng.randint(1, 64)
        P = _log_int(rng, 16, max(16, min(MOST_ROWS, MOST_SCORES // (M * Hq)) - M))
        return {"kind": kind, "fmt": fmt, "M": M, "P": P, "Hq": Hq, "Hkv": Hkv, "pad": rng.randint(1, M - 1) if M > 3 and rng.random() < 0.25 else 0}
    M = _log_int(rng, 1, 60)
    return {"kind": kind, "M": M, "V": _log_int(rng, 1000, 128256), "filters": rng.choice(["none", "k", "p", "kp", "min", "all"]),
            "banned": rng.random() < 0.3}


# ---- inputs ----------------------------------------------------------------------------------------------


def _normal(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(torch.float16)


def _keys(gen, rows, Hkv, D):
    """rows of a key or value cache: unit normal, a few channels of each head several times as wide"""
    wide = 1 + 5 * (torch.rand(Hkv, D, generator=gen, device=DEV) < 0.03)
    return (torch.randn(rows, Hkv, D, generator=gen, device=DEV) * wide).to(torch.float16)


def _chain_or_tree(seed, M, pad):
    """ancestor mask uint8 [M, M] and depths of a draft: a chain up to 8 rows, else a random tree; the last `pad` rows are no nodes"""
    rng = np.random.default_rng(seed)
    n = M - pad
    parent = [-1] + [i - 1 if n <= 8 else int(rng.integers(max(0, (i - 1) // 4), i)) for i in range(1, n)]
    mask, depth = np.zeros((M, M), dtype=np.uint8), np.zeros(M, dtype=np.int64)
    for i in range(n):
        if i:
            mask[i], depth[i] = mask[parent[i]], depth[parent[i]] + 1
        mask[i, i] = 1
    return torch.from_numpy(mask).to(DEV), torch.from_numpy(depth).to(DEV)


def _tables(n_pos, D):
    """fp32 cos and sin [n_pos, D / 2] of position p times 500000^(-2 i / D)"""
    ang = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * 500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=DEV) / D)
    return ang.cos().float(), ang.sin().float()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    half = lambda *shape: torch.empty(*shape, dtype=torch.float16, device=DEV)
    if kind == "append":
        M, P, Hq, Hkv, D = (case[n] for n in ("M", "P", "Hq", "Hkv", "D"))
        s["qkv"] = _normal(gen, M, (Hq + 2 * Hkv) * D, std=2.0)
        s["gq"], s["gk"] = (1 + _normal(gen, D, std=0.2), 1 + _normal(gen, D, std=0.2)) if case["norm"] else (None, None)
        if M <= 64:
            _, depth = _chain_or_tree(seed, M, 0)
        else:
            depth = torch.arange(M, device=DEV)
        s["pos"] = (P + depth).to(torch.int32)
        s["cos"], s["sin"] = _tables(P + M, D)
        s["q"] = half(M, Hq, D)
        rows = P + M
        if case["fmt"] == "fp16":
            s["k"], s["v"] = _keys(gen, rows, Hkv, D), _keys(gen, rows, Hkv, D)
        else:
            s["k"], s["ks"] = _quantise(_keys(gen, rows, Hkv, D), case["fmt"])
            s["v"], s["vs"] = _quantise(_keys(gen, rows, Hkv, D), case["fmt"])
            s["k_out"], s["v_out"] = half(M, Hkv, D), half(M, Hkv, D)
    elif kind == "read":
        rows, first, Hkv, D = (case[n] for n in ("rows", "first", "Hkv", "D"))
        s["k"], s["ks"] = _quantise(_keys(gen, first + rows + 5, Hkv, D), case["fmt"])
        s["v"], s["vs"] = _quantise(_keys(gen, first + rows + 5, Hkv, D), case["fmt"])
        s["k_out"], s["v_out"] = half(rows, Hkv, D), half(rows, Hkv, D)
    elif kind == "attn":
        M, P, Hq, Hkv = (case[n] for n in ("M", "P", "Hq", "Hkv"))
        s["q"] = _normal(gen, M, Hq, D_ATTN, std=1.2)
        s["k"], s["ks"] = _quantise(_keys(gen, P + M, Hkv, D_ATTN), case["fmt"])
        s["v"], s["vs"] = _quantise(_keys(gen, P + M, Hkv, D_ATTN), case["fmt"])
        s["mask"], _ = _chain_or_tree(seed, M, case["pad"])
        s["out"] = half(M, Hq, D_ATTN)
    else:
        M, V, f = case["M"], case["V"], case["filters"]
        rand = lambda *shape: torch.rand(*shape, generator=gen, device=DEV)
        s["logits"] = 2.2 * torch.randn(M, V, generator=gen, device=DEV) + 12 * rand(M, V) ** 200
        if case["banned"]:
            s["logits"].masked_fill_(rand(M, V) < 0.2, -math.inf)
        s["temperature"] = 0.5 + rand(M)
        if M > 4:
            s["temperature"][1] = 0.0     # one request of the batch decodes greedily
        s["top_k"] = torch.randint(5, 200, (M,), generator=gen, device=DEV, dtype=torch.int32) if f in ("k", "kp", "all") else None
        s["top_p"] = 0.7 + 0.29 * rand(M) if f in ("p", "kp", "all") else None
        s["min_p"] = 0.1 * rand(M) if f in ("min", "all") else None
        s["u"] = rand(M)
        s["token"] = torch.empty(M, dtype=torch.int32, device=DEV)
        s["prob"] = torch.empty(M, dtype=torch.float32, device=DEV)
    if own:   # scratch memory that a program allocates once
        from paper_2505_22179_amd import binding as B
        if kind == "attn":
            s["ws"] = B.new_workspace(B.tree_verify_attn_kv8_workspace_bytes(M, P, Hq, Hkv, D_ATTN))
        elif kind == "sample":
            s["ws"] = B.new_workspace(B.lm_head_sample_workspace_bytes(M, V))
    return s


# ---- plain forms -----------------------------------------------------------------------------------------


def _quantise(x, fmt):
    """codes [rows, heads, D] and fp16 scales [rows, heads] of fp16 x"""
    amax = x.abs().amax(-1).double()     # in 64 bits a quotient that is a scale itself stays one, whatever way the division is done
    if fmt == "int8":
        t = (amax / 127.0).float()
        four = ((t.view(torch.int32) + 0xFFFFF) & ~0xFFFFF).view(torch.float32)       # up to four significant bits
        scale = torch.where(t < 2.0 ** -21, torch.ceil(t * 2.0 ** 24).clamp(min=1) * 2.0 ** -24, four).clamp(max=512.0)
        codes = torch.round(x / scale[..., None]).clamp(-127, 127).to(torch.int8)
    else:
        t = (amax / 448.0).float()
        scale = ((t.view(torch.int32) + 0x7FFFFF) & ~0x7FFFFF).view(torch.float32).clamp(min=2.0 ** -15)
        most = torch.where(scale == 256.0, 240.0, 448.0)[..., None]                   # 256 * 256 is beyond fp16
        codes = torch.minimum(torch.maximum(x / scale[..., None], -most), most).to(torch.float8_e4m3fn)
    return codes, scale.to(torch.float16)


def _values(codes, scales):
    return codes.float() * scales.float()[..., None]


def _append(s):
    case = s["case"]
    M, P, Hq, Hkv, D, fmt = (case[n] for n in ("M", "P", "Hq", "Hkv", "D", "fmt"))
    x = s["qkv"].view(M, Hq + 2 * Hkv, D)
    v = x[:, Hq + Hkv:]
    qk = x[:, :Hq + Hkv].float()
    if case["norm"]:
        gamma = torch.cat([s["gq"].float().expand(Hq, D), s["gk"].float().expand(Hkv, D)])
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS) * gamma
    c, n = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    a, b = qk[..., :D // 2], qk[..., D // 2:]
    qk = torch.cat([a * c - b * n, b * c + a * n], -1).to(torch.float16)
    q, k = qk[:, :Hq], qk[:, Hq:]
    if fmt == "fp16":
        s["k"][P:P + M], s["v"][P:P + M] = k, v
        return q, s["k"], s["v"]
    (kc, ks), (vc, vs) = _quantise(k, fmt), _quantise(v, fmt)
    s["k"][P:P + M], s["ks"][P:P + M], s["v"][P:P + M], s["vs"][P:P + M] = kc, ks, vc, vs
    return q, _values(kc, ks).to(torch.float16), _values(vc, vs).to(torch.float16)


def _attend(s):
    case = s["case"]
    M, P, Hq, Hkv = (case[n] for n in ("M", "P", "Hq", "Hkv"))
    group, T = Hq // Hkv, P + M
    q = s["q"].float().view(M, Hkv, group, D_ATTN).permute(1, 2, 0, 3).reshape(Hkv, group * M, D_ATTN)
    k = _values(s["k"], s["ks"]).permute(1, 2, 0).contiguous()
    v = _values(s["v"], s["vs"]).permute(1, 0, 2).contiguous()
    hidden = torch.cat([torch.zeros(M, P, dtype=torch.bool, device=DEV), s["mask"] == 0], 1)
    hidden = hidden | ~s["mask"].bool().any(1)[:, None] if case["pad"] else hidden   # rows behind the tree see nothing at all
    scores = (torch.matmul(q, k) * D_ATTN ** -0.5).view(Hkv, group, M, T).masked_fill(hidden, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = torch.matmul(p.view(Hkv, group * M, T), v)
    return out.view(Hkv, group, M, D_ATTN).permute(2, 0, 1, 3).reshape(M, Hq, D_ATTN).to(torch.float16)


def _sample(s):
    M, V = s["logits"].shape
    x, order = torch.sort(s["logits"].double(), dim=1, descending=True, stable=True)   # equal logits in token order
    T = s["temperature"].double()[:, None]
    greedy = T <= 0
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, 1.0, T))
    rank = torch.arange(V, device=DEV)[None]
    k = s["top_k"].long()[:, None] if s["top_k"] is not None else torch.full((M, 1), V, device=DEV)
    w = torch.where(rank < torch.where(greedy, 1, torch.where(k > 0, k, V)), w, 0.0)
    if s["top_p"] is not None:
        before = torch.cumsum(w, 1) - w
        p = s["top_p"].double()[:, None]
        w = torch.where((before < p * w.sum(1, keepdim=True)) | (p >= 1) | (rank == 0), w, 0.0)
    if s["min_p"] is not None:
        w = torch.where((w >= s["min_p"].double()[:, None]) | (rank == 0), w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)
    total = torch.cumsum(w, 1)
    token = (total <= s["u"].double()[:, None] * total[:, -1:]).sum(1, keepdim=True)
    token = torch.minimum(token, torch.where(w > 0, rank, 0).amax(1, keepdim=True))
    return token[:, 0].to(torch.int32), (w.gather(1, token) / total[:, -1:])[:, 0].float()


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, case, kind)
    if kind == "append":
        return _append(s)
    if kind == "read":
        at = slice(case["first"], case["first"] + case["rows"])
        return _values(s["k"][at], s["ks"][at]).to(torch.float16), _values(s["v"][at], s["vs"][at]).to(torch.float16)
    return _attend(s) if kind == "attn" else _sample(s)


def _run_own(s, case, kind):
    from paper_2505_22179_amd import binding as B
    if kind == "sample":
        B.lm_head_sample(s["logits"], case["M"], case["V"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"], s["token"], s["prob"], s["ws"])
        return s["token"], s["prob"]
    if kind == "append" and case["fmt"] == "fp16":
        M, P, Hq, Hkv, D = (case[n] for n in ("M", "P", "Hq", "Hkv", "D"))
        B.rope_append_qk_norm(s["qkv"], s["gq"], s["gk"], EPS, s["pos"], s["cos"], s["sin"], P + M, s["q"], s["k"], s["v"], M, P, Hq, Hkv, D)
        return s["q"], s["k"], s["v"]
    fmt = B.KV8_INT8 if case["fmt"] == "int8" else B.KV8_E4M3
    if kind == "append":
        M, P, Hq, Hkv, D = (case[n] for n in ("M", "P", "Hq", "Hkv", "D"))
        B.rope_append_kv8(s["qkv"], s["gq"], s["gk"], EPS, s["pos"], s["cos"], s["sin"], P + M, s["q"], s["k"], s["v"], s["ks"], s["vs"], fmt,
                     M, P, Hq, Hkv, D)
        B.w4a16_kv8_read(s["k"], s["v"], s["ks"], s["vs"], fmt, P, M, Hkv, D, s["k_out"], s["v_out"])   # the values that the codes stand for
        return s["q"], s["k_out"], s["v_out"]
    if kind == "read":
        B.w4a16_kv8_read(s["k"], s["v"], s["ks"], s["vs"], fmt, case["first"], case["rows"], case["Hkv"], case["D"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    B.tree_verify_attn_kv8(s["q"], s["k"], s["v"], s["ks"], s["vs"], fmt, s["mask"], s["out"], case["M"], case["P"], case["Hq"], case["Hkv"],
                           D_ATTN, D_ATTN ** -0.5, s["ws"])
    return s["out"]


# ---- bytes and operations that a pass cannot do without ----------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "append":
        M, P, Hq, Hkv, D = (case[n] for n in ("M", "P", "Hq", "Hkv", "D"))
        heads, cached = Hq + 2 * Hkv, 2 * M * Hkv
        bytes_ = 2 * M * heads * D + 4 * M + 4 * M * D + 2 * M * Hq * D + (4 * D if case["norm"] else 0)
        bytes_ += 2 * cached * D if case["fmt"] == "fp16" else cached * (D + 2) + 2 * cached * D    # codes and scales, and the values read back
        return {"bytes": bytes_, "flops": M * (Hq + Hkv) * D * (3.0 + (4.0 if case["norm"] else 0.0)) + (4.0 * cached * D if case["fmt"] != "fp16" else 0.0)}
    if kind == "read":
        n = 2 * case["rows"] * case["Hkv"]
        return {"bytes": n * (case["D"] + 2) + 2 * n * case["D"], "flops": 1.0 * n * case["D"]}
    if kind == "attn":
        M, P, Hq, Hkv = (case[n] for n in ("M", "P", "Hq", "Hkv"))
        return {"bytes": 4 * M * Hq * D_ATTN + 2 * (P + M) * Hkv * (D_ATTN + 2) + M * M, "flops": 4.0 * (M - case["pad"]) * (P + M) * Hq * D_ATTN}
    M, V = case["M"], case["V"]
    return {"bytes": 4 * M * V + 28 * M, "flops": 4.0 * M * V}


# ---- the same in 64 bits -----------------------------------------------------------------------------------


def _power(e):
    """2^e in 64 bits, exactly (torch.ldexp goes through a power in 32 bits)"""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _stored64(x, fmt):
    """what an 8-bit cache holds of x (float64 tensor, rounded to fp16 first), by the definition"""
    x = x.to(torch.float16).double()
    amax = x.abs().amax(-1, keepdim=True)
    if fmt == "int8":
        mant, exp = torch.frexp(amax / 127)                       # amax / 127 = mant 2^exp, mant in [1/2, 1)
        unit = _power(torch.clamp(exp - 4, min=-24))
        s = torch.clamp(torch.ceil(amax / 127 / unit), min=1) * unit
        s = torch.clamp(s, max=512)
        return torch.clamp(torch.round(x / s), -127, 127) * s
    mant, exp = torch.frexp(amax / 448)
    e = torch.clamp(torch.where(mant == 0.5, exp - 1, exp), min=-15)
    s = _power(e)
    y = x / s
    most = torch.where(e == 8, 240.0, 448.0).double()
    y = torch.maximum(torch.minimum(y, most), -most)
    _, ye = torch.frexp(y)
    step = _power(torch.clamp(ye - 4, min=-9))   # three bits behind the leading one, 2^-9 at the least
    return torch.round(y / step) * step * s


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "append":
        M, P, Hq, Hkv, D = (case[n] for n in ("M", "P", "Hq", "Hkv", "D"))
        x = s["qkv"].double().view(M, -1, D)

        def turned(y, gamma):
            if gamma is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + EPS) * gamma.double()
            at = s["pos"].long()
            turn = torch.complex(s["cos"].double()[at], s["sin"].double()[at])[:, None]
            z = torch.complex(y[..., :D // 2].contiguous(), y[..., D // 2:].contiguous()) * turn
            return torch.cat([z.real, z.imag], -1)

        q, k, v = turned(x[:, :Hq], s["gq"]), turned(x[:, Hq:Hq + Hkv], s["gk"]), x[:, Hq + Hkv:]
        if case["fmt"] != "fp16":
            return q, _stored64(k, case["fmt"]), _stored64(v, case["fmt"])
        all_k, all_v = s["k"].double(), s["v"].double()
        all_k[P:P + M], all_v[P:P + M] = k, v
        return q, all_k, all_v
    if kind == "read":
        at = slice(case["first"], case["first"] + case["rows"])
        return tuple(c[at].to(torch.float32).double() * t[at].double().unsqueeze(-1) for c, t in ((s["k"], s["ks"]), (s["v"], s["vs"])))
    if kind == "attn":
        M, P, Hq, Hkv = (case[n] for n in ("M", "P", "Hq", "Hkv"))
        out = torch.zeros(M, Hq, D_ATTN, dtype=torch.float64, device=DEV)
        nodes = M - case["pad"]
        seen = torch.cat([torch.ones(nodes, P, dtype=torch.bool, device=DEV), s["mask"][:nodes] != 0], 1)
        for g in range(Hkv):
            k, v = (c[:, g].to(torch.float32).double() * t[:, g].double()[:, None] for c, t in ((s["k"], s["ks"]), (s["v"], s["vs"])))
            k = k.t().contiguous()
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                a = (s["q"][:nodes, h].double() @ k) / math.sqrt(D_ATTN)
                out[:nodes, h] = torch.softmax(torch.where(seen, a, -math.inf), 1) @ v
        return out
    # token by token in numpy; the token itself is a whole number and has no value here beyond its probability
    prob = []
    host = lambda t, fill: np.full(case["M"], fill) if t is None else t.cpu().numpy().astype(np.float64)
    rows, T, K, Pp, Mp, u = s["logits"].cpu().numpy().astype(np.float64), host(s["temperature"], 1), host(s["top_k"], 0), host(s["top_p"], 1), host(s["min_p"], 0), host(s["u"], 0)
    for m in range(case["M"]):
        if T[m] <= 0:
            prob.append(1.0)
            continue
        order = np.argsort(-rows[m], kind="stable")
        if K[m] > 0:
            order = order[:int(K[m])]
        w = np.exp((rows[m][order] - rows[m].max()) / T[m])
        if Pp[m] < 1:
            order = order[:max(1, int(np.searchsorted(np.concatenate([[0.0], np.cumsum(w)[:-1]]), Pp[m] * w.sum(), side="left")))]
            w = w[:len(order)]
        n = max(1, int((w >= Mp[m]).sum()))
        order, w = order[:n], w[:n]
        by_token = np.argsort(order)
        at = min(int(np.searchsorted(np.cumsum(w[by_token]), u[m] * w.sum(), side="right")), n - 1)
        prob.append(w[by_token[at]] / w.sum())
    return None, torch.tensor(prob, dtype=torch.float64)
