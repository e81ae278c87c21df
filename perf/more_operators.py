"""Operators that take a prompt, or a batch of sequences of different lengths, through a layer whose weights and activations have 8 bits, and what
one pass through each has to return:

  table    cos and sin of the rotary embedding for a range of positions, scaled for long contexts
  rope     rotation of the queries and keys of packed tokens (half or interleaved pairs, the whole head or the first part of it), keys and
           values scattered to the cache rows that a slot map names
  linear   x -> int8 codes with a scale for each token; their product with an int8 weight that has a scale for each channel. x is taken as it
           is, normed, or as silu(gate) * up; a residual may be added
  attn     causal attention of packed sequences of different lengths: the queries of a sequence are the last of its keys. One query each
           is a batch of decode steps

Without `own` a pass is elementary torch operations in 32 bits (64 for the angles and for the quotients that decide a code).
Definitions shared by both:
  table    f_i = theta^(-2 i / R); n_i = original f_i / (2 pi), the turns of pair i within the original context
           linear: f / factor.  turns: t f + (1 - t) f / factor with t = (n - low) / (high - low) within [0, 1]
           index:  r f / factor + (1 - r) f with r = (i - a) / (b - a) within [0, 1], a and b the pairs that turn `high` and `low` times,
           a rounded down and at least 0, b rounded up and at most R - 1;  entries amplitude cos(p f), amplitude sin(p f)
  linear   s = max|x| / 127 in fp32, code = x / s rounded to the nearest (ties to even), y = sum code w  s  t (+ residual), rounded once; what a norm
           or a gate gives is rounded to fp16 before it is quantised"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-5
HEADS = [(32, 8), (64, 8), (40, 8), (16, 2), (12, 2), (8, 8), (28, 4)]
MOST_MACS = 8192 * 28672 * 4096            # of a linear
MOST_SCORES = 16384 * 16384 // 2 * 32      # visible (query, key, head) triples of an attention
MOST_TABLE = 131072 * 128


def listed():
    return [
        # the tables of a short context that a program makes when it starts; a quarter of each head is turned
        {"name": "table_4096_r32", "kind": "table", "first": 0, "n": 4096, "R": 32, "theta": 10000.0, "scaling": "none", "factor": 1.0},
        # those of the longest context, stretched eightfold
        {"name": "table_131072_r128_turns", "kind": "table", "first": 0, "n": 131072, "R": 128, "theta": 500000.0, "scaling": "turns", "factor": 8.0},
        # one decode step of a batch: 16 sequences, 8B heads, latency is all there is
        {"name": "rope_m16", "kind": "rope", "M": 16, "n_pos": 8192, "Hq": 32, "Hkv": 8, "D": 128, "R": 128, "interleaved": False},
        # a batch of prompts, 70B heads, interleaved pairs
        {"name": "rope_m8192_interleaved", "kind": "rope", "M": 8192, "n_pos": 8192, "Hq": 64, "Hkv": 8, "D": 128, "R": 128, "interleaved": True},
        # plain decoding: one normed token through an 8B gate and up projection, bound by the weights
        {"name": "linear_m1_norm", "kind": "linear", "M": 1, "N": 28672, "K": 4096, "pre": "norm", "residual": False},
        # a verified tree of 60 nodes through a 70B o projection, residual
        {"name": "linear_m60_residual", "kind": "linear", "M": 60, "N": 8192, "K": 8192, "pre": "plain", "residual": True},
        # a short prompt of odd length through an 8B down projection, gate and residual
        {"name": "linear_m777_silu", "kind": "linear", "M": 777, "N": 4096, "K": 14336, "pre": "silu", "residual": True},
        # a large batch of prompts through an 8B gate and up projection: the most arithmetic
        {"name": "linear_m8192_norm", "kind": "linear", "M": 8192, "N": 28672, "K": 4096, "pre": "norm", "residual": False},
        # decode steps of 16 sequences of ragged lengths, 8B heads: bound by the cache
        {"name": "attn_decode_b16_k8192", "kind": "attn", "B": 16, "n": 1, "prefix": 8191, "Hq": 32, "Hkv": 8, "D": 128, "pad": 0},
        # many short prompts packed, heads of 64, rows behind the last one
        {"name": "attn_b24_n700_d64", "kind": "attn", "B": 24, "n": 700, "prefix": 0, "Hq": 28, "Hkv": 4, "D": 64, "pad": 5},
        # the next piece of a long prompt behind what the cache holds, 70B heads
        {"name": "attn_n509_k30000", "kind": "attn", "B": 1, "n": 509, "prefix": 29491, "Hq": 64, "Hkv": 8, "D": 128, "pad": 3},
        # one long prompt, 8B heads: the most arithmetic
        {"name": "attn_n16384", "kind": "attn", "B": 1, "n": 16384, "prefix": 0, "Hq": 32, "Hkv": 8, "D": 128, "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["table", "rope", "linear", "linear", "attn", "attn", "attn"])
    if kind == "table":
        R = 2 * rng.randint(8, 64)
        scaling = rng.choice(["none", "linear", "turns", "index"])
        return {"kind": kind, "first": rng.choice([0, 0, rng.randint(1, 10000)]), "n": _log_int(rng, 1, min(131072, MOST_TABLE // R)), "R": R,
                "theta": rng.choice([10000.0, 500000.0, 1000000.0]), "scaling": scaling, "factor": 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0])}
    Hq, Hkv = rng.choice(HEADS)
    if kind == "rope":
        D = rng.choice([64, 80, 96, 128, 128, 256])
        M = _log_int(rng, 1, min(8192, 8192 * 80 * 128 // ((Hq + 2 * Hkv) * D)))
        return {"kind": kind, "M": M, "n_pos": max(M, _log_int(rng, 256, 16384)), "Hq": Hq, "Hkv": Hkv, "D": D, "R": rng.choice([D, D, D // 2, D // 4]),
                "interleaved": rng.random() < 0.5}
    if kind == "linear":
        N, K = 8 * _log_int(rng, 32, 3584), 16 * _log_int(rng, 16, 896)
        return {"kind": kind, "M": _log_int(rng, 1, min(8192, MOST_MACS // (N * K))), "N": N, "K": K, "pre": rng.choice(["plain", "norm", "silu"]),
                "residual": rng.random() < 0.5}
    D = rng.choice([64, 128, 128])
    form = rng.choice(["decode", "prompts", "piece"])
    B = _log_int(rng, 1, 64) if form != "piece" else rng.randint(1, 3)
    if form == "decode":
        n, prefix = rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 16, min(65536, 1 << 24) // max(1, B * Hkv // 64))
    elif form == "prompts":
        n, prefix = _log_int(rng, 1, int(math.sqrt(2 * MOST_SCORES / (B * Hq)))), 0
    else:
        n = _log_int(rng, 8, 2048)
        prefix = _log_int(rng, 16, max(16, min(65536, MOST_SCORES // (B * Hq * n))))
    return {"kind": kind, "B": B, "n": min(n, 16384), "prefix": prefix, "Hq": Hq, "Hkv": Hkv, "D": D, "pad": rng.choice([0, 0, 1, 7])}


def _lengths(case):
    """(queries, keys) of each sequence: the first is the longest, the others are spread below it"""
    rng = random.Random("%d %d %d" % (case["B"], case["n"], case["prefix"]))
    n = [case["n"]] + [_log_int(rng, 1, case["n"]) for _ in range(case["B"] - 1)]
    before = [case["prefix"]] + [_log_int(rng, 1, case["prefix"]) if case["prefix"] else 0 for _ in range(case["B"] - 1)]
    return [(a, a + b) for a, b in zip(n, before)]


# ---- inputs ----------------------------------------------------------------------------------------------


def _normal(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(torch.float16)


def _keys(gen, rows, Hkv, D):
    """rows of a key or value cache: unit normal, a few channels of each head several times as wide"""
    wide = 1 + 5 * (torch.rand(Hkv, D, generator=gen, device=DEV) < 0.03)
    return (torch.randn(rows, Hkv, D, generator=gen, device=DEV) * wide).to(torch.float16)


def _hidden(gen, rows, K):
    """activations: unit normal, a few channels ten times as wide, as hidden states of large models have them"""
    wide = 1 + 9 * (torch.rand(K, generator=gen, device=DEV) < 0.005)
    return (torch.randn(rows, K, generator=gen, device=DEV) * wide).to(torch.float16)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    half = lambda *shape: torch.empty(*shape, dtype=torch.float16, device=DEV)
    if kind == "table":
        s["cos"], s["sin"] = (torch.empty(case["n"], case["R"] // 2, device=DEV) for _ in range(2))
        # base and trained context as the seed has them; 1 + a tenth of the logarithm of the stretch
        s["theta"], s["original"] = case["theta"] * (1 + (seed % 97) / 97), 8192.0 - 64.0 * (seed % 32)
        s["amplitude"] = 1.0 + 0.1 * math.log(case["factor"]) if case["scaling"] == "index" else 1.0
    elif kind == "rope":
        M, n_pos, Hq, Hkv, D, R = (case[n] for n in ("M", "n_pos", "Hq", "Hkv", "D", "R"))
        s["qkv"] = _normal(gen, M, (Hq + 2 * Hkv) * D, std=1.5)
        s["pos"] = torch.randint(0, n_pos, (M,), generator=gen, device=DEV, dtype=torch.int32)
        s["rows"] = M + M // 4 + 3      # the batch's tokens lie in blocks of the cache, some of whose rows are other sequences'
        starts = torch.randperm((s["rows"] + 15) // 16, generator=gen, device=DEV)
        slots = (starts[:, None] * 16 + torch.arange(16, device=DEV)[None]).reshape(-1)
        s["slot"] = slots[slots < s["rows"]][:M].to(torch.int32)
        if M > 3:
            s["slot"][M // 2] = -1      # a padding token
        ang = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * 500000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device=DEV) / R)
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        s["q"], s["k"], s["v"] = half(M, Hq, D), _normal(gen, s["rows"], Hkv, D), _normal(gen, s["rows"], Hkv, D)
    elif kind == "linear":
        M, N, K = (case[n] for n in ("M", "N", "K"))
        s["x"] = _hidden(gen, M, K) if case["pre"] != "silu" else _normal(gen, M, 2 * K, std=1.2)
        s["gamma"] = 1 + _normal(gen, K, std=0.2) if case["pre"] == "norm" else None
        s["w"] = torch.clamp(torch.round(torch.randn(N, K, generator=gen, device=DEV) * 30), -127, 127).to(torch.int8)
        s["t"] = (0.5 + torch.rand(N, generator=gen, device=DEV)) / (30 * math.sqrt(K))
        s["residual"] = _normal(gen, M, N) if case["residual"] else None
        s["y"] = half(M, N)
    else:
        Hq, Hkv, D = (case[n] for n in ("Hq", "Hkv", "D"))
        s["lens"] = _lengths(case)
        rows = sum(n for n, _ in s["lens"])
        q_start, k_start, at, row = [], [], 0, 0
        for n, k in s["lens"]:      # a whole prompt's keys lie as its queries do; a cache has gaps between sequences
            q_start.append(at)
            k_start.append(row)
            at, row = at + n, row + k + (16 if case["prefix"] else 0)
        s["at"] = list(zip(q_start, k_start))
        s["q"], s["k"], s["v"] = _normal(gen, rows + case["pad"], Hq, D, std=1.2), _keys(gen, row, Hkv, D), _keys(gen, row, Hkv, D)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        s["q_start"], s["k_start"], s["k_len"] = ints(q_start + [rows]), ints(k_start), ints([k for _, k in s["lens"]])
        s["out"] = torch.zeros(rows + case["pad"], Hq, D, dtype=torch.float16, device=DEV)
    if own:   # the weight laid out once, scratch memory that a program allocates once
        from paper_2505_22179_amd import binding as B
        if kind == "linear":
            s["packed"] = torch.empty(B.w8a8_packed_bytes(N, K), dtype=torch.uint8, device=DEV)
            B.w8a8_pack(s["w"], s["packed"], N, K)
            s["ws"] = B.new_workspace(B.w8a8_workspace_bytes(M, N, K))
        elif kind == "attn":
            s["most"] = case["n"], case["n"] + case["prefix"]
            s["ws"] = B.new_workspace(B.w4a16_prompt_attn_workspace_bytes(s["q"].shape[0], case["B"], *s["most"], Hq, Hkv, D))
    return s


# ---- plain forms -----------------------------------------------------------------------------------------

LOW, HIGH = {"turns": 1.0, "index": 1.0}, {"turns": 4.0, "index": 32.0}


def _table(s):
    case = s["case"]
    R, theta, scaling, factor = case["R"], s["theta"], case["scaling"], case["factor"]
    i = torch.arange(R // 2, dtype=torch.float64, device=DEV)
    f = theta ** (-2 * i / R)
    if scaling == "linear":
        f = f / factor
    elif scaling == "turns":
        t = ((s["original"] * f / (2 * math.pi) - LOW[scaling]) / (HIGH[scaling] - LOW[scaling])).clamp(0, 1)
        f = t * f + (1 - t) * f / factor
    elif scaling == "index":
        pair = lambda turns: R * math.log(s["original"] / (turns * 2 * math.pi)) / (2 * math.log(theta))
        a, b = max(math.floor(pair(HIGH[scaling])), 0), min(math.ceil(pair(LOW[scaling])), R - 1)
        r = ((i - a) / max(b - a, 0.001)).clamp(0, 1)
        f = r * f / factor + (1 - r) * f
    ang = torch.arange(case["first"], case["first"] + case["n"], dtype=torch.float64, device=DEV)[:, None] * f
    return (ang.cos() * s["amplitude"]).float(), (ang.sin() * s["amplitude"]).float()


def _rope(s):
    case = s["case"]
    M, Hq, Hkv, D, R = (case[n] for n in ("M", "Hq", "Hkv", "D", "R"))
    x = s["qkv"].view(M, Hq + 2 * Hkv, D)
    turned = x[:, :Hq + Hkv].float()
    c, n = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    if case["interleaved"]:
        a, b = turned[..., 0:R:2], turned[..., 1:R:2]
        part = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = turned[..., :R // 2], turned[..., R // 2:R]
        part = torch.cat([a * c - b * n, b * c + a * n], -1)
    qk = torch.cat([part, turned[..., R:]], -1).to(torch.float16)
    stored = s["slot"] >= 0
    to = s["slot"][stored].long()
    s["k"][to], s["v"][to] = qk[:, Hq:][stored], x[:, Hq + Hkv:][stored]
    return qk[:, :Hq], s["k"], s["v"]


def _linear(s):
    case = s["case"]
    x = s["x"].float()
    if case["pre"] == "norm":
        x = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s["gamma"].float()).to(torch.float16)
    elif case["pre"] == "silu":
        gate, up = x[:, :case["K"]], x[:, case["K"]:]
        x = (gate / (1 + torch.exp(-gate)) * up).to(torch.float16)
    x = x.double()
    scale = (x.abs().amax(-1, keepdim=True) / 127).float()
    codes = torch.round(x / scale.double()).float()
    y = torch.matmul(codes, s["w"].float().t()) * scale * s["t"]
    return (y + s["residual"].float() if case["residual"] else y).to(torch.float16)


def _attend(s):
    case = s["case"]
    Hq, Hkv, D = (case[n] for n in ("Hq", "Hkv", "D"))
    group = Hq // Hkv
    for (n, T), (at, row) in zip(s["lens"], s["at"]):
        q = s["q"][at:at + n].float().view(n, Hkv, group, D).permute(1, 2, 0, 3).reshape(Hkv, group * n, D)
        k = s["k"][row:row + T].float().permute(1, 2, 0).contiguous()
        v = s["v"][row:row + T].float().permute(1, 0, 2).contiguous()
        hidden = torch.arange(T, device=DEV)[None] > torch.arange(T - n, T, device=DEV)[:, None]
        heads = max(1, min(Hkv, (1 << 29) // (group * n * T)))      # heads at a time
        for h in range(0, Hkv, heads):
            here = slice(h, min(h + heads, Hkv))
            scores = (torch.matmul(q[here], k[here]) * D ** -0.5).view(-1, group, n, T).masked_fill_(hidden, -math.inf)
            p = torch.exp_(scores.sub_(scores.amax(-1, keepdim=True)))
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(-1, group * n, T), v[here]).view(-1, group, n, D) / total
            s["out"][at:at + n].view(n, Hkv, group, D)[:, here] = o.permute(2, 0, 1, 3).to(torch.float16)
    return s["out"]


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, s["case"], kind)
    return _table(s) if kind == "table" else _rope(s) if kind == "rope" else _linear(s) if kind == "linear" else _attend(s)


def _run_own(s, case, kind):
    from paper_2505_22179_amd import binding as B
    if kind == "table":
        scaling = {"none": B.ROPE_PLAIN, "linear": B.ROPE_LINEAR, "turns": B.ROPE_BY_TURNS, "index": B.ROPE_BY_INDEX}[case["scaling"]]
        B.rope_table(s["cos"], s["sin"], case["first"], case["n"], case["R"], s["theta"], scaling, case["factor"], LOW.get(case["scaling"], 0.0),
                     HIGH.get(case["scaling"], 0.0), s["original"], s["amplitude"])
        return s["cos"], s["sin"]
    if kind == "rope":
        B.rope_prompt(s["qkv"], s["pos"], s["cos"], s["sin"], case["n_pos"], case["R"], case["interleaved"], s["slot"], s["rows"], s["q"], s["k"], s["v"],
                      case["M"], case["Hq"], case["Hkv"], case["D"])
        return s["q"], s["k"], s["v"]
    if kind == "linear":
        pre = {"plain": B.W8A8_PLAIN, "norm": B.W8A8_RMS_NORM, "silu": B.W8A8_SILU_MUL}[case["pre"]]
        B.w8a8_linear(s["x"], pre, s["gamma"], EPS, s["packed"], s["t"], s["residual"], s["y"], case["M"], case["N"], case["K"], s["ws"])
        return s["y"]
    B.w4a16_prompt_attn(s["q"], s["k"], s["v"], s["q_start"], s["k_start"], s["k_len"], s["out"], case["B"], s["q"].shape[0], s["k"].shape[0], *s["most"],
                        case["Hq"], case["Hkv"], case["D"], case["D"] ** -0.5, s["ws"])
    return s["out"]


# ---- bytes and operations that a pass cannot do without ----------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "table":
        return {"bytes": 4 * case["n"] * case["R"], "flops": 1.0 * case["n"] * case["R"]}
    if kind == "rope":
        M, Hq, Hkv, D, R = (case[n] for n in ("M", "Hq", "Hkv", "D", "R"))
        return {"bytes": 4 * M * (Hq + 2 * Hkv) * D + 8 * M + 4 * R * min(M, case["n_pos"]), "flops": 3.0 * M * (Hq + Hkv) * R}
    if kind == "linear":
        M, N, K = (case[n] for n in ("M", "N", "K"))
        return {"bytes": N * K + 4 * N + 2 * M * K * (2 if case["pre"] == "silu" else 1) + 2 * M * N * (2 if case["residual"] else 1), "flops": 2.0 * M * N * K}
    lens = _lengths(case)
    rows, seen = sum(n for n, _ in lens), sum(n * T - n * (n - 1) // 2 for n, T in lens)
    return {"bytes": 4 * rows * case["Hq"] * case["D"] + 4 * sum(T for _, T in lens) * case["Hkv"] * case["D"], "flops": 4.0 * seen * case["Hq"] * case["D"]}


# ---- the same in 64 bits -----------------------------------------------------------------------------------


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "table":
        R, turn = case["R"], 2 * math.pi
        f = []
        for i in range(R // 2):
            plain = math.exp(-math.log(s["theta"]) * 2 * i / R)
            near, far = plain, plain / case["factor"]      # as trained, and stretched
            if case["scaling"] == "none":
                f.append(near)
            elif case["scaling"] == "linear":
                f.append(far)
            elif case["scaling"] == "turns":
                share = (s["original"] * plain / turn - 1.0) / 3.0
                f.append(near if share >= 1 else far if share <= 0 else share * near + (1 - share) * far)
            else:
                first, last = (R / 2 * math.log(s["original"] / (m * turn), s["theta"]) for m in (32.0, 1.0))
                first, last = max(0, math.floor(first)), min(R - 1, math.ceil(last))
                share = min(1.0, max(0.0, (i - first) / ((last - first) or 0.001)))
                f.append(share * far + (1 - share) * near)
        at = torch.arange(case["n"], dtype=torch.float64, device=DEV) + case["first"]
        z = torch.polar(torch.full((case["n"], R // 2), s["amplitude"], dtype=torch.float64, device=DEV), torch.outer(at, torch.tensor(f, dtype=torch.float64, device=DEV)))
        return z.real.clone(), z.imag.clone()
    if kind == "rope":
        M, Hq, Hkv, D, R = (case[n] for n in ("M", "Hq", "Hkv", "D", "R"))
        x = s["qkv"].double().view(M, -1, D)
        pairs = torch.arange(R, device=DEV).view(-1, 2) if case["interleaved"] else torch.arange(R, device=DEV).view(2, -1).t()
        turn = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()].unsqueeze(1)
        z = torch.complex(x[:, :Hq + Hkv, pairs[:, 0]], x[:, :Hq + Hkv, pairs[:, 1]]) * turn
        x[:, :Hq + Hkv, pairs[:, 0]], x[:, :Hq + Hkv, pairs[:, 1]] = z.real, z.imag
        k, v = s["k"].double(), s["v"].double()
        for m, to in enumerate(s["slot"].tolist()) if M <= 64 else ():
            if to >= 0:
                k[to], v[to] = x[m, Hq:Hq + Hkv], x[m, Hq + Hkv:]
        if M > 64:
            ok = torch.nonzero(s["slot"] >= 0)[:, 0]
            k.index_copy_(0, s["slot"][ok].long(), x[ok, Hq:Hq + Hkv])
            v.index_copy_(0, s["slot"][ok].long(), x[ok, Hq + Hkv:])
        return x[:, :Hq], k, v
    if kind == "linear":
        x = s["x"].double()
        if case["pre"] == "norm":
            x = x / torch.sqrt((x * x).sum(1, keepdim=True) / case["K"] + EPS) * s["gamma"].double()
        elif case["pre"] == "silu":
            gate, up = x.chunk(2, 1)
            x = gate * torch.sigmoid(gate) * up
        x = x.to(torch.float16).double()
        scale = (x.abs().max(1).values / 127).to(torch.float32).double()
        codes = torch.round(x / scale[:, None])
        y = torch.empty(case["M"], case["N"], dtype=torch.float64, device=DEV)
        for n in range(0, case["N"], 4096):
            y[:, n:n + 4096] = codes @ s["w"][n:n + 4096].double().t()
        y *= torch.outer(scale, s["t"].double())
        return y if s["residual"] is None else y + s["residual"].double()
    out = s["out"].double()
    if work(case)["flops"] > 1.5e13:
        return None
    for (n, T), (at, row) in zip(s["lens"], s["at"]):
        for h in range(case["Hq"]):
            g = h // (case["Hq"] // case["Hkv"])
            k, v = (c[row:row + T, g].double() for c in (s["k"], s["v"]))
            kt = k.t().contiguous()
            for lo in range(0, n, 2048):
                hi = min(n, lo + 2048)
                a = s["q"][at + lo:at + hi, h].double() @ kt / math.sqrt(case["D"])
                a += torch.full((hi - lo, T), -math.inf, dtype=torch.float64, device=DEV).triu(T - n + lo + 1)
                out[at + lo:at + hi, h] = torch.softmax(a, 1) @ v
    return out
