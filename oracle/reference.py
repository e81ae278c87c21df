"""Python face of the CPU oracle.  TEST INFRASTRUCTURE ONLY: imported by tests/, by the smoke
check and by the benchmark's cpu_baseline leg, never by the product package.

Linear layer (paper section 2.2, W4A16 with group size 128): thin ctypes wrappers around the C
file next to this one, which carries the definition (unpack, exact fp32 dequantisation, fp32
k-ascending sum with an fp64 shadow, round-to-nearest-even fp16).

Tree-verify attention (paper section 2.1: the target model scores all n draft-tree tokens in one
forward pass; a draft token may attend to the committed prefix, to itself and to its ancestors in
the tree): plain numpy in fp64, written below.

Greedy tree acceptance and K/V compaction (the integer step right after verification): plain
Python below; pinned in tests/test_oracle_accept.py by brute force over all root paths, chain
closed forms, planted paths and library gathers.

Layer glue (RMS norm, residual and SiLU-gate epilogues of the linears, rotary embedding with K/V
append): plain numpy in fp64 at the end of this file; pinned in tests/test_oracle_layer.py by
closed forms, one-hot inputs that reduce the linear to a table lookup, rotation invariants and the
torch library routines.

Draft-side LM head with log-softmax and top-k: numpy fp64 at the end of this file; pinned in
tests/test_oracle_lm_head.py (one-hot rows, planted winners, probabilities that sum to one, ties,
torch's log_softmax / topk).

Pin status.  The paper prints no worked numerical example for any of these operations, so beyond the
pins in tests/test_oracle_*.py (nibble-order fixtures, round trips, closed forms, exact rational
brute force, numpy/torch library cross-checks, structural invariants) the numerics are unpinned
by the paper and this oracle is the definition.
"""
from __future__ import annotations

import ctypes
import math
import os

import numpy as np

from . import build as _build

_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        path = _build.build()
        L = ctypes.CDLL(path)
        vp, i = ctypes.c_void_p, ctypes.c_int
        L.orc_f16_to_f32.restype = ctypes.c_float
        L.orc_f16_to_f32.argtypes = [ctypes.c_uint16]
        L.orc_f32_to_f16.restype = ctypes.c_uint16
        L.orc_f32_to_f16.argtypes = [ctypes.c_float]
        L.orc_f16_to_f32_array.argtypes = [vp, vp, ctypes.c_size_t]
        L.orc_f32_to_f16_array.argtypes = [vp, vp, ctypes.c_size_t]
        L.orc_unpack_codes.argtypes = [vp, vp, i, i]
        L.orc_unpack_zeros.argtypes = [vp, vp, i, i]
        L.orc_dequant.argtypes = [vp, vp, vp, vp, i, i, i]
        L.orc_matmul.argtypes = [vp, vp, vp, vp, vp, i, i, i]
        L.orc_gemm.argtypes = [vp] * 8 + [i] * 4
        L.orc_set_threads.restype = i
        L.orc_set_threads.argtypes = [i]
        for name in ("orc_f16_to_f32_array", "orc_f32_to_f16_array", "orc_unpack_codes",
                     "orc_unpack_zeros", "orc_dequant", "orc_matmul", "orc_gemm"):
            getattr(L, name).restype = None
        _lib = L
    return _lib


def _p(a: np.ndarray) -> ctypes.c_void_p:
    assert a.flags["C_CONTIGUOUS"]
    return ctypes.c_void_p(a.ctypes.data)


def set_threads(n: int) -> int:
    """n > 0 sets the OpenMP thread count; returns the count in effect."""
    return int(lib().orc_set_threads(int(n)))


def f16_to_f32(h: np.ndarray) -> np.ndarray:
    h = np.ascontiguousarray(h).view(np.uint16)
    out = np.empty(h.shape, dtype=np.float32)
    lib().orc_f16_to_f32_array(_p(h), _p(out), h.size)
    return out


def f32_to_f16(f: np.ndarray) -> np.ndarray:
    f = np.ascontiguousarray(f, dtype=np.float32)
    out = np.empty(f.shape, dtype=np.uint16)
    lib().orc_f32_to_f16_array(_p(f), _p(out), f.size)
    return out.view(np.float16)


def unpack_codes(qweight: np.ndarray) -> np.ndarray:
    """int32 [K/8, N] -> uint8 [K, N]"""
    qweight = np.ascontiguousarray(qweight, dtype=np.int32)
    K, N = qweight.shape[0] * 8, qweight.shape[1]
    q = np.empty((K, N), dtype=np.uint8)
    lib().orc_unpack_codes(_p(qweight), _p(q), K, N)
    return q


def unpack_zeros(qzeros: np.ndarray) -> np.ndarray:
    """int32 [K/G, N/8] -> uint8 [K/G, N]"""
    qzeros = np.ascontiguousarray(qzeros, dtype=np.int32)
    R, N = qzeros.shape[0], qzeros.shape[1] * 8
    z = np.empty((R, N), dtype=np.uint8)
    lib().orc_unpack_zeros(_p(qzeros), _p(z), R, N)
    return z


def dequant(qweight: np.ndarray, scales: np.ndarray, qzeros: np.ndarray, G: int = 128) -> np.ndarray:
    """-> fp32 [K, N], w = (q - z) * s, exact"""
    qweight = np.ascontiguousarray(qweight, dtype=np.int32)
    qzeros = np.ascontiguousarray(qzeros, dtype=np.int32)
    scales = np.ascontiguousarray(scales, dtype=np.float16)
    K, N = qweight.shape[0] * 8, qweight.shape[1]
    assert scales.shape == (K // G, N) and qzeros.shape == (K // G, N // 8)
    W = np.empty((K, N), dtype=np.float32)
    lib().orc_dequant(_p(qweight), _p(scales.view(np.uint16)), _p(qzeros), _p(W), N, K, G)
    return W


def matmul(x: np.ndarray, W: np.ndarray, want64: bool = True):
    """x fp16 [M, K], W fp32 [K, N] -> (y32, y64 or None, y16)"""
    x = np.ascontiguousarray(x, dtype=np.float16)
    W = np.ascontiguousarray(W, dtype=np.float32)
    M, K = x.shape
    N = W.shape[1]
    assert W.shape[0] == K
    y32 = np.empty((M, N), dtype=np.float32)
    y64 = np.empty((M, N), dtype=np.float64) if want64 else None
    y16 = np.empty((M, N), dtype=np.uint16)
    lib().orc_matmul(_p(x.view(np.uint16)), _p(W), _p(y32), _p(y64) if want64 else None, _p(y16), M, N, K)
    return y32, y64, y16.view(np.float16)


def w4a16_gemm(x, qweight, scales, qzeros, G: int = 128, want64: bool = True):
    """The whole layer: returns (y32, y64 or None, y16)."""
    W = dequant(qweight, scales, qzeros, G)
    return matmul(x, W, want64)


# ---------------------------------------------------------------------------------------------
# tree-verify attention, fp64


def tree_verify_attn(q, k, v, mask, scale: float | None = None):
    """q fp16 [M, Hq, D]; k, v fp16 [P+M, Hkv, D]; mask [M, M] (non-zero = visible).
    Query row i of head h attends, through KV head h // (Hq/Hkv), to all P prefix keys and to the
    draft keys j with mask[i, j] != 0.  Returns (out64 [M, Hq, D] fp64, out16 fp16)."""
    q = np.asarray(q)
    k = np.asarray(k)
    v = np.asarray(v)
    mask = np.asarray(mask)
    M, Hq, D = q.shape
    T, Hkv, _ = k.shape
    P = T - M
    assert P >= 0 and mask.shape == (M, M) and Hq % Hkv == 0
    if scale is None:
        scale = 1.0 / np.sqrt(D)
    rep = Hq // Hkv
    q64, k64, v64 = q.astype(np.float64), k.astype(np.float64), v.astype(np.float64)
    out = np.zeros((M, Hq, D), dtype=np.float64)
    for i in range(M):
        visible = np.concatenate([np.ones(P, dtype=bool), mask[i] != 0])
        for h in range(Hq):
            kh = h // rep
            logits = scale * (k64[visible, kh, :] @ q64[i, h, :])
            logits -= logits.max()
            p = np.exp(logits)
            p /= p.sum()
            out[i, h, :] = p @ v64[visible, kh, :]
    return out, out.astype(np.float16)


# ---------------------------------------------------------------------------------------------
# greedy acceptance of a verified draft tree and compaction of the accepted K/V rows


def tree_accept(parent, token, target):
    """Greedy draft-then-verify acceptance on a tree draft (paper section 2.1: the target model
    verifies the n draft-tree tokens in one pass and accepts some of them; section 4: verifying a
    tree turns it into a sequence).  Node 0 is the root, i.e. the last committed token; parent[i] < i.
    token[i] is the draft token at node i, target[i] the target model's greedy next token after
    the sequence ending in node i.  The walk starts at the root; at node cur, a child is accepted
    iff its draft token equals target[cur]; among several such children the lowest index is taken;
    the walk stops at the first node without an accepted child.
    Returns (path, next_token): the accepted node indices, root first, and target[path[-1]], the
    token the target model itself contributes after the last accepted node.  Pure integer work."""
    parent = [int(p) for p in parent]
    token = [int(t) for t in token]
    target = [int(t) for t in target]
    n = len(parent)
    assert n >= 1 and parent[0] < 0 and all(0 <= parent[i] < i for i in range(1, n))
    path = [0]
    cur = 0
    while True:
        nxt = -1
        for i in range(cur + 1, n):
            if parent[i] == cur and token[i] == target[cur]:
                nxt = i
                break
        if nxt < 0:
            break
        path.append(nxt)
        cur = nxt
    return path, target[cur]


def kv_compact(k, v, path, P: int):
    """After acceptance the cache keeps the accepted nodes only, in order: cache row P + j receives
    the K and V rows of node path[j] (stored at row P + path[j]) for every j < len(path).  Rows
    below P and rows from P + len(path) on are left as they are.  Returns new arrays."""
    k2, v2 = np.array(k, copy=True), np.array(v, copy=True)
    for j, node in enumerate(path):
        k2[P + j] = k[P + node]
        v2[P + j] = v[P + node]
    return k2, v2


# ---------------------------------------------------------------------------------------------
# the other steps of a decoder layer around the four linears (paper section 2.1: one target-model
# forward pass over the draft tokens is the unit of cost T_v(n); the target is a Llama-3 model, whose
# layer is  h += Wo.attn(rope(Wqkv.norm(h)));  h += Wdown.(silu(Wgate.norm(h)) * Wup.norm(h)) ).
# All in fp64 from the fp16 inputs, one rounding to fp16 at the end of each function.


def silu(v):
    """v * sigmoid(v) = v / (1 + exp(-v)), fp64"""
    v = np.asarray(v, dtype=np.float64)
    return v / (1.0 + np.exp(-v))


def rms_norm(x, gamma, eps: float):
    """x fp16 [M, K], gamma fp16 [K] -> (y64, y16):  y[m,k] = x[m,k] * gamma[k] / sqrt(mean_k x[m,:]^2 + eps)"""
    x64 = np.asarray(x).astype(np.float64)
    g64 = np.asarray(gamma).astype(np.float64)
    ms = (x64 * x64).sum(axis=1, keepdims=True) / x64.shape[1]
    y = x64 * g64[None, :] / np.sqrt(ms + float(eps))
    return y, y.astype(np.float16)


def w4a16_gemm_residual(x, qweight, scales, qzeros, residual, G: int = 128):
    """(y64, y16):  y = residual + x . W   (the o_proj and down projections add into the hidden state)"""
    _, y64, _ = w4a16_gemm(x, qweight, scales, qzeros, G, want64=True)
    y = y64 + np.asarray(residual).astype(np.float64)
    return y, y.astype(np.float16)


def w4a16_gemm_silu_mul(x, qweight, scales, qzeros, G: int = 128):
    """(y64, y16) of shape [M, N/2]: columns 0..N/2-1 of the weight are the gate projection, columns
    N/2..N-1 the up projection;  y[m,n] = silu(x.W[:, n]) * (x.W[:, N/2 + n])"""
    _, y64, _ = w4a16_gemm(x, qweight, scales, qzeros, G, want64=True)
    half = y64.shape[1] // 2
    assert 2 * half == y64.shape[1]
    y = silu(y64[:, :half]) * y64[:, half:]
    return y, y.astype(np.float16)


def rope_append(qkv, pos, cos, sin, k_cache, v_cache, P: int, Hq: int, Hkv: int, D: int):
    """Rotary position embedding of the q and k parts of a fused projection output and the append of
    the new keys and values to the cache.
    qkv fp16 [M, (Hq + 2 Hkv) D]: per row Hq query heads, then Hkv key heads, then Hkv value heads;
    pos int [M]: position of each row (for a draft tree: prefix length + depth of the node);
    cos, sin fp32 [n_pos, D/2]: caller's tables, entry [p, i] belongs to position p and the pair of
    head elements (i, i + D/2):  out[i] = a[i] cos - a[i + D/2] sin,  out[i + D/2] = a[i + D/2] cos + a[i] sin.
    Returns (q64 [M, Hq, D], q16, k_cache', v_cache') where rows P..P+M-1 of the fp16 caches
    [>= P+M, Hkv, D] hold the rotated keys and the unchanged values; other rows are untouched."""
    qkv = np.asarray(qkv)
    M = qkv.shape[0]
    assert qkv.shape[1] == (Hq + 2 * Hkv) * D and D % 2 == 0
    a = qkv.astype(np.float64).reshape(M, Hq + 2 * Hkv, D)
    c = np.asarray(cos).astype(np.float64)[np.asarray(pos)][:, None, :]   # [M, 1, D/2]
    s = np.asarray(sin).astype(np.float64)[np.asarray(pos)][:, None, :]
    h = D // 2

    def rot(t):
        lo, hi = t[..., :h], t[..., h:]
        return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)

    q = rot(a[:, :Hq])
    k = rot(a[:, Hq:Hq + Hkv])
    k2, v2 = np.array(k_cache, copy=True), np.array(v_cache, copy=True)
    k2[P:P + M] = k.astype(np.float16)
    v2[P:P + M] = qkv.reshape(M, Hq + 2 * Hkv, D)[:, Hq + Hkv:]
    return q, q.astype(np.float16), k2, v2


# ---------------------------------------------------------------------------------------------
# draft side: fp16 language-model head, log-softmax and top-k (paper section 2.1: the draft model
# uses the target's LM head and expands its beam search by the softmax output; section 3.1: the
# draft stays in fp16 because LM head and softmax are its bottleneck and are not quantisable)


def lm_head_topk(x, W, top_k: int):
    """x fp16 [M, K] (draft hidden states), W fp16 [V, K] (LM-head weight, one row per token).
    logits[m, v] = sum_k x[m, k] W[v, k];  logprob = logits - log(sum_v exp(logits)), per row.
    Returns (logits64 [M, V], idx int64 [M, top_k], logprob64 [M, top_k]): per row the top_k tokens by
    logit, largest first, equal logits in ascending token order, with their log-probabilities."""
    x64 = np.asarray(x).astype(np.float64)
    W64 = np.asarray(W).astype(np.float64)
    logits = x64 @ W64.T
    mx = logits.max(axis=1, keepdims=True)
    lse = mx[:, 0] + np.log(np.exp(logits - mx).sum(axis=1))
    M, V = logits.shape
    idx = np.empty((M, top_k), dtype=np.int64)
    for m in range(M):
        order = sorted(range(V), key=lambda v: (-logits[m, v], v))   # plain definition of the order
        idx[m] = order[:top_k]
    lp = np.take_along_axis(logits, idx, axis=1) - lse[:, None]
    return logits, idx, lp


# ---------------------------------------------------------------------------------------------
# head norms ahead of the rotation, and the 8-bit attention cache


def rope_append_qk_norm(qkv, q_gamma, k_gamma, eps: float, pos, cos, sin, k_cache, v_cache, P: int, Hq: int, Hkv: int, D: int):
    """rope_append with every query and key head x replaced by x * gamma / sqrt(mean(x^2) + eps) first.  fp64; returns
    (q, k_cache, v_cache) like rope_append, unrounded (float64 arrays)."""
    x = np.array(qkv, dtype=np.float64).reshape(len(pos), Hq + 2 * Hkv, D)
    for first, last, gamma in ((0, Hq, q_gamma), (Hq, Hq + Hkv, k_gamma)):
        part = x[:, first:last]
        x[:, first:last] = part / np.sqrt((part * part).mean(-1, keepdims=True) + eps) * np.asarray(gamma, dtype=np.float64)
    half = D // 2
    c, s = (np.asarray(t, dtype=np.float64)[np.asarray(pos)][:, None, :] for t in (cos, sin))
    a, b = x[:, :Hq + Hkv, :half].copy(), x[:, :Hq + Hkv, half:].copy()
    x[:, :Hq + Hkv, :half] = a * c - b * s
    x[:, :Hq + Hkv, half:] = b * c + a * s
    k2, v2 = np.array(k_cache, dtype=np.float64), np.array(v_cache, dtype=np.float64)
    k2[P:P + len(pos)] = x[:, Hq:Hq + Hkv]
    v2[P:P + len(pos)] = x[:, Hq + Hkv:]
    return x[:, :Hq], k2, v2


INT8, E4M3 = 1, 2


def e4m3_table():
    """the numbers of the 256 e4m3 codes (sign, four exponent bits of bias 7, three mantissa bits; 0x7F and 0xFF are NaN)"""
    out = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        mag = np.nan if code & 0x7F == 0x7F else (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        out[code] = -mag if code & 0x80 else mag
    return out


def _nearest_e4m3(y):
    """codes of the e4m3 numbers nearest to y (|y| <= 448), ties to the even mantissa; zeros keep their sign"""
    grid = e4m3_table()[:0x7F]                       # 0 .. 448, increasing
    mag = np.abs(y)
    hi = np.clip(np.searchsorted(grid, mag, side="left"), 1, 0x7E)
    lo = hi - 1
    below, above = mag - grid[lo], grid[hi] - mag     # exact: the operands are short
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def kv8_quantise(x, fmt: int):
    """codes uint8 [..., D] (int8 codes as their bytes) and scales fp16 [...] of fp16 x [..., D], by the definition of the format.
    The scale is found in whole numbers of 2^-24, of which every fp16 number is one."""
    x = np.asarray(x, dtype=np.float16)
    codes, scales = np.zeros(x.shape, dtype=np.uint8), np.full(x.shape[:-1], np.nan, dtype=np.float16)
    for at in np.ndindex(*x.shape[:-1]):
        row = x[at].astype(np.float64)
        if not np.isfinite(row).all():
            continue                                  # codes 0, scale NaN
        units = int(np.abs(row).max() * 2.0 ** 24)
        if fmt == INT8:
            want = -(-units // 127)                   # ceil
            shift = max(0, want.bit_length() - 4)
            want = -(-units // (127 << shift)) << shift
            if want.bit_length() > shift + 4:         # 15.x rounded up to 16: one bit more
                want = -(-units // (127 << (shift + 1))) << (shift + 1)
            s = min(max(want, 1) * 2.0 ** -24, 512.0)
            codes[at] = np.clip(np.rint(row / s), -127, 127).astype(np.int8).view(np.uint8)
        else:
            s = 2.0 ** -15
            while s * 448 < units * 2.0 ** -24:
                s *= 2
            most = 240.0 if s == 256 else 448.0
            codes[at] = _nearest_e4m3(np.clip(row / s, -most, most))
        scales[at] = s
    return codes, scales


def kv8_values(codes, scales, fmt: int):
    """float64 values of codes and scales"""
    numbers = np.asarray(codes).view(np.int8).astype(np.float64) if fmt == INT8 else e4m3_table()[np.asarray(codes)]
    return numbers * np.asarray(scales, dtype=np.float64)[..., None]


def tree_verify_attn_seen(q, k, v, mask, scale: float):
    """tree_verify_attn for trees padded to a fixed size and caches whose hidden rows may hold anything: a row whose mask row is empty is
    padding, sees nothing, committed keys included, and gets zeros.
    Returns (out, spread) in float64, spread = sum_j p_j |v_j| (what the rounding of the probabilities acts on)."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    M, Hq, D = q.shape
    T, Hkv, _ = k.shape
    P = T - M
    out, spread = np.zeros((M, Hq, D)), np.zeros((M, Hq, D))
    for i in range(M):
        draft = np.asarray(mask)[i] != 0
        seen = np.flatnonzero(np.concatenate([np.ones(P, dtype=bool), draft]))
        for g in range(Hkv if draft.any() else 0):
            heads = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
            with np.errstate(invalid="ignore"):
                logits = scale * (q[i, heads] @ k[seen, g].T)
                p = np.exp(logits - logits.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                out[i, heads] = p @ v[seen, g]
                spread[i, heads] = p @ np.abs(v[seen, g])
    return out, spread


# ---------------------------------------------------------------------------------------------
# sampling from the logits of a language-model head


def sample(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """One row.  Returns (token, probability, margin): the token and its share of the kept weight, by the definition in include/w4a16.h, and
    how near a border decided -- the smallest distance, as a share of the row's weight, between u or top_p and a cumulative weight next to it, or
    between min_p and a weight.  Plain Python over the tokens in order."""
    x = [float(v) for v in logits]
    order = sorted((v for v in range(len(x)) if x[v] > -math.inf), key=lambda v: (-x[v], v))   # NaN compares false
    if not order:
        return 0x7FFFFFFF, 0.0, 1.0
    top = x[order[0]]
    if not temperature > 0 or top_p <= 0 or min_p > 1:
        return order[0], 1.0, 1.0
    weight = lambda v: 1.0 if x[v] == top else 0.0 if math.isinf(top) else math.exp((x[v] - top) / temperature)
    if 0 < top_k < len(order):
        order = order[:top_k]
    w = {v: weight(v) for v in order}
    margin, total = 1.0, math.fsum(w.values())
    if top_p < 1:
        kept, before = [], 0.0
        for v in order:
            if kept and w[v] > 0:
                margin = min(margin, abs(before / total - top_p))
            if kept and not before < top_p * total:
                break
            kept.append(v)
            before += w[v]
        order = kept
    if min_p > 0:
        margin = min([margin] + [abs(w[v] - min_p) for v in order[1:]])
        order = order[:1] + [v for v in order[1:] if w[v] >= min_p]
    order = sorted(v for v in order if w[v] > 0)
    total, upto = math.fsum(w[v] for v in order), 0.0
    for v in order:
        upto += w[v]
        margin = min(margin, abs(upto / total - u)) if v != order[-1] else margin
        if upto > u * total or v == order[-1]:
            return v, w[v] / total, margin


# ---------------------------------------------------------------------------------------------
# prompts: rotary tables for long contexts, rotation with scatter, W8A8 linears, causal attention of packed sequences


def rope_frequencies(R, theta, scaling=0, factor=1.0, low=0.0, high=0.0, original=0.0):
    """float64 [R / 2], by the formulas in include/w4a16.h"""
    out = []
    for i in range(R // 2):
        f = float(theta) ** (-2.0 * i / R)
        if scaling == 1:
            f /= factor
        elif scaling == 2:
            t = min(max((original * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = t * f + (1 - t) * f / factor
        elif scaling == 3:
            index = lambda turns: R * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))
            a, b = max(float(math.floor(index(high))), 0.0), min(float(math.ceil(index(low))), R - 1.0)
            r = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f = r * f / factor + (1 - r) * f
        out.append(f)
    return np.array(out)


def rope_table(first, n_pos, R, theta, scaling=0, factor=1.0, low=0.0, high=0.0, original=0.0, amplitude=1.0):
    """(cos, sin) float64 [n_pos, R / 2]"""
    ang = np.arange(first, first + n_pos, dtype=np.float64)[:, None] * rope_frequencies(R, theta, scaling, factor, low, high, original)
    return amplitude * np.cos(ang), amplitude * np.sin(ang)


def rope_prompt(qkv, pos, cos, sin, R, interleaved, slot, q, k_cache, v_cache):
    """(q, k_cache, v_cache) float64, exact: copies of the given ones with what rope_prompt writes"""
    q, k_cache, v_cache = (np.asarray(t, dtype=np.float64).copy() for t in (q, k_cache, v_cache))
    rows, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    x = np.asarray(qkv, dtype=np.float64).reshape(rows, Hq + 2 * Hkv, D)
    for m in range(rows):
        to = m if slot is None else int(slot[m])
        stored = 0 <= to < k_cache.shape[0]
        if stored:
            v_cache[to] = x[m, Hq + Hkv:]
        if not 0 <= pos[m] < cos.shape[0]:
            continue
        y = x[m, :Hq + Hkv].copy()
        for i in range(R // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
            c, s = float(cos[pos[m], i]), float(sin[pos[m], i])
            y[:, a], y[:, b] = x[m, :Hq + Hkv, a] * c - x[m, :Hq + Hkv, b] * s, x[m, :Hq + Hkv, b] * c + x[m, :Hq + Hkv, a] * s
        q[m] = y[:Hq]
        if stored:
            k_cache[to] = y[Hq:]
    return q, k_cache, v_cache


def w8a8_input(x, pre, gamma=None, eps=0.0):
    """float64: what a W8A8 linear quantises, before its rounding to fp16"""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if pre == 1:
            return x * np.asarray(gamma, dtype=np.float64) / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if pre == 2:
            gate, up = np.split(x, 2, axis=-1)
            return gate / (1 + np.exp(-gate)) * up
    return x


def w8a8_quantise(x16):
    """(codes int8, scales float32) of fp16 rows; the quotient is rounded exactly (ties to even): x / s in float64 cannot come as near to a half
    that it is not without being one (x has 11 bits, s 24, the code 8)"""
    x = np.asarray(x16, dtype=np.float64)
    top = np.abs(x).max(-1)
    fine = np.isfinite(x).all(-1)
    scale = np.where(fine, np.float32(np.where(fine, top, 0.0) / 127), np.float32(np.nan)).astype(np.float32)
    s = np.where(fine & (top > 0), scale, 1).astype(np.float64)[..., None]
    codes = np.rint(np.where((fine & (top > 0))[..., None], x, 0.0) / s).astype(np.int8)
    return codes, scale


def w8a8_gemm(codes, scale, w, w_scale, residual=None):
    """float64 [M, N], exact but for float64's own roundings: integer sums"""
    acc = np.asarray(codes, dtype=np.int64) @ np.asarray(w, dtype=np.int64).T
    y = acc * np.asarray(scale, dtype=np.float64)[:, None] * np.asarray(w_scale, dtype=np.float64)
    return y if residual is None else y + np.asarray(residual, dtype=np.float64)


def w8a8_layout(codes, fill=0):
    """codes [rows, K] in the layout of include/w8a8.h; rows of the padding hold `fill`"""
    rows, K = codes.shape
    R, KP = (rows + 15) // 16 * 16, (K + 127) // 128 * 128
    full = np.zeros((R, KP), dtype=np.int8)
    full[:rows, :K], full[rows:] = codes, fill
    return np.ascontiguousarray(full.reshape(R // 16, 16, KP // 64, 4, 16).transpose(0, 2, 3, 1, 4)).reshape(-1)


def prompt_attn(q, k, v, q_start, k_start, k_len, scale, out):
    """(out, spread) float64: `out` with the rows of the sequences replaced; spread = sum_j p_j |v_j| of those rows"""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    out, spread = np.asarray(out, dtype=np.float64).copy(), np.zeros(q.shape)
    group = q.shape[1] // k.shape[1]
    for b in range(len(q_start) - 1):
        q0, q1 = int(q_start[b]), int(q_start[b + 1])
        k0, T = (q0, q1 - q0) if k_len is None else (int(k_start[b]), int(k_len[b]))
        if q0 < 0 or q1 > q.shape[0] or k0 < 0 or T < 0 or k0 + T > k.shape[0]:
            continue
        for i in range(q0, q1):
            seen = T - (q1 - q0) + (i - q0) + 1
            out[i], spread[i] = 0.0, 0.0
            if seen <= 0:
                continue
            with np.errstate(invalid="ignore"):
                for h in range(q.shape[1]):
                    a = scale * (k[k0:k0 + seen, h // group] @ q[i, h])
                    p = np.exp(a - a.max())
                    p /= p.sum()
                    out[i, h], spread[i, h] = p @ v[k0:k0 + seen, h // group], p @ np.abs(v[k0:k0 + seen, h // group])
    return out, spread
