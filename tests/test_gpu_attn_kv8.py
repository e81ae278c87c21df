"""GPU: tree_verify_attn_kv8 through the C ABI against the fp64 oracle over the values of the cache.

Tolerance per output, derived: probabilities are rounded to fp16 (2^-11 of each, 2^-25 below 2^-14; 128-row sums of products in fp32 stay far below
that), a score errs by the fp32 sum of 128 products, at most 128 2^-24 sum |q k| times the scale, which moves each weight by that
share, and twice so with the normalisation; the output is rounded once (2^-11 of it)."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import binding as B
from paper_2505_22179_amd import inputs as I

pytestmark = pytest.mark.gpu
DEV, D = "cuda", 128
dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
FORMATS = [B.KV8_INT8, B.KV8_E4M3]


class Call:
    def __init__(self, seed, M, P, Hq, Hkv, fmt, tree="random", q_std=1.0, v_std=1.0, scale=None):
        rng = np.random.default_rng(seed)
        self.M, self.P, self.Hq, self.Hkv, self.fmt = M, P, Hq, Hkv, fmt
        self.scale = scale or D ** -0.5
        self.q = (rng.standard_normal((M, Hq, D)) * q_std).astype(np.float16)
        T = P + M
        if fmt == B.KV8_INT8:
            codes = lambda: np.clip(np.rint(rng.standard_normal((T, Hkv, D)) * 40), -127, 127).astype(np.int8).view(np.uint8)
            scales = lambda std: (rng.integers(8, 16, (T, Hkv)) * 2.0 ** (-9 + rng.integers(0, 3, (T, Hkv))) * std).astype(np.float16)
        else:
            codes = lambda: R._nearest_e4m3(np.clip(rng.standard_normal((T, Hkv, D)) * 100, -448, 448))
            scales = lambda std: (2.0 ** (-8 + rng.integers(0, 3, (T, Hkv))) * std).astype(np.float16)
        self.k, self.ks, self.v, self.vs = codes(), scales(1.0), codes(), scales(v_std)
        if tree == "random" and M > 1:
            self.mask = I.make_tree(seed + 1, M, min(6, M - 1), 4)[2]
        else:
            self.mask = I.chain_tree(M)[2] if tree == "chain" or M == 1 else np.eye(M, dtype=np.uint8)

    def tensors(self):
        return [dev(t) for t in (self.q, self.k, self.v, self.ks, self.vs)] + [self.fmt, dev(self.mask)]

    def sizes(self):
        return self.M, self.P, self.Hq, self.Hkv, D, self.scale

    def workspace(self):
        return B.new_workspace(B.tree_verify_attn_kv8_workspace_bytes(self.M, self.P, self.Hq, self.Hkv, D))

    def run(self, ws=None):
        out = torch.full((self.M + 1, self.Hq, D), 77.0, dtype=torch.float16, device=DEV)
        B.tree_verify_attn_kv8(*self.tensors(), out, *self.sizes(), self.workspace() if ws is None else ws)
        torch.cuda.synchronize()
        o = out.cpu().numpy()
        assert (o[self.M:] == 77).all()
        return o[:self.M]

    def check(self, out16):
        k, v = R.kv8_values(self.k, self.ks, self.fmt), R.kv8_values(self.v, self.vs, self.fmt)
        want, spread = R.tree_verify_attn_seen(self.q, k, v, self.mask, self.scale)
        np.testing.assert_array_equal(np.isnan(out16), np.isnan(want))
        rep = self.Hq // self.Hkv
        with np.errstate(invalid="ignore"):
            qk = np.nanmax(np.abs(self.q.astype(np.float64)).sum(-1)) * np.nanmax(np.abs(k)) * self.scale   # above every sum |q k| scale
            score = 2 * 128 * 2.0 ** -24 * min(qk, 64.0 * 8)
            vmax = np.nanmax(np.abs(v), axis=(0, 2)).repeat(rep)[None, :, None]
            tol = spread * (2.0 ** -11 * 1.01 + score) + np.abs(want) * 2.0 ** -11 + 2.0 ** -25 + (self.P + self.M) * 2.0 ** -25 * vmax / max(1.0, (self.P + self.M) ** 0.5)
            err = np.abs(out16.astype(np.float64) - want)
        worst = np.nanmax(err / tol)
        assert worst <= 1, f"worst error {worst:.3g} of the tolerance"
        fine = ~np.isnan(want)
        rel = np.linalg.norm((out16 - want)[fine]) / max(np.linalg.norm(want[fine]), 1e-30)
        assert rel <= 2.0 ** -10, rel
        return rel


CASES = [
    # M, P, Hq, Hkv, tree
    (1, 2048, 64, 8, "chain"),       # plain decoding
    (1, 0, 8, 1, "chain"),           # a single key
    (1, 30, 8, 8, "chain"),          # 31 keys: one short of a step
    (1, 31, 8, 8, "chain"),          # exactly one step
    (1, 32, 7, 1, "chain"),
    (7, 2048, 32, 8, "chain"),       # sequence verification
    (60, 2048, 64, 8, "random"),     # tree verification
    (64, 100, 8, 8, "random"),
    (64, 64, 64, 8, "random"),       # 512 rows per KV head
    (17, 0, 16, 4, "random"),        # no prefix
    (33, 31, 8, 2, "identity"),
    (48, 5, 4, 1, "random"),
    (3, 2, 12, 2, "chain"),          # fewer keys than one step
    (12, 300, 32, 4, "random"),
    (37, 1333, 28, 4, "random"),     # groups of seven
    (5, 70, 40, 8, "random"),        # groups of five
    (8, 10001, 16, 2, "random"),     # many steps per range, ragged end
    (40, 5000, 8, 1, "random"),      # one KV head: 320 rows over a long prefix
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,P,Hq,Hkv,tree", CASES)
def test_parity(M, P, Hq, Hkv, tree, fmt):
    print(f"attn_kv8 parity M={M} P={P} Hq={Hq} Hkv={Hkv} {tree} fmt={fmt}", flush=True)
    c = Call(3000 + M + P + Hq, M, P, Hq, Hkv, fmt, tree)
    out = c.run()
    c.check(out)
    np.testing.assert_array_equal(c.run().view(np.uint16), out.view(np.uint16))   # the same bits again


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("v_std", [2.0 ** -6, 16.0])
def test_values_of_any_size(fmt, v_std):
    """scales near both ends: codes times scale stay fp16 numbers, nothing under- or overflows on the way"""
    c = Call(11, 9, 700, 16, 4, fmt, v_std=v_std)
    c.check(c.run())


@pytest.mark.parametrize("fmt", FORMATS)
def test_sharp_softmax(fmt):
    """large scores: a few keys carry everything, running maxima move from step to step"""
    c = Call(12, 20, 3000, 16, 4, fmt, q_std=6.0)
    c.check(c.run())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,P,Hq,Hkv", [(9, 0, 16, 4), (37, 250, 28, 4), (64, 33, 64, 8), (60, 0, 8, 1)])
def test_rows_that_see_nothing_and_hidden_rows_that_hold_anything(M, P, Hq, Hkv, fmt):
    """a tree padded to a fixed size: the last rows are no nodes -- with no prefix they see nothing -- and their cache rows were never written"""
    print(f"attn_kv8 padded M={M} P={P} Hq={Hq} Hkv={Hkv} fmt={fmt}", flush=True)
    c = Call(50 + M, M, P, Hq, Hkv, fmt)
    n = M - M // 3
    c.mask[n:], c.mask[:, n:] = 0, 0
    clean = c.run()
    c.check(clean)
    assert P or (clean[n:] == 0).all()
    rng = np.random.default_rng(M)
    for codes, scales in ((c.k, c.ks), (c.v, c.vs)):
        codes[P + n:] = rng.choice(np.array([0x7F, 0xFF, 0x80, 0x7E], dtype=np.uint8), codes[P + n:].shape)
        scales[P + n:] = rng.choice(np.array([np.nan, np.inf, -np.inf, 65504.0, 1.0], dtype=np.float16), scales[P + n:].shape)
    np.testing.assert_array_equal(c.run().view(np.uint16), clean.view(np.uint16))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("at", [3, 70, 100])
def test_a_nan_key_or_value_reaches_the_rows_that_see_it_and_no_others(at, fmt):
    """NaN scales: at a committed row all query rows see it; at a draft row only its descendants"""
    M, P = 12, 96
    for which in ("ks", "vs"):
        c = Call(60 + at, M, P, 8, 2, fmt, tree="random")
        getattr(c, which)[at, 1] = np.nan
        getattr(c, which[0])[at, 1] = 0     # as rope_append_kv8 writes it
        out = c.run()
        c.check(out)
        assert not np.isnan(out[:, :4]).any() and np.isnan(out[:, 4:]).any()


@pytest.mark.parametrize("fmt", FORMATS)
def test_infinite_and_nan_queries_stay_in_their_rows(fmt):
    c = Call(61, 10, 200, 8, 2, fmt)
    clean = c.run()
    c.q[4, 3, 7], c.q[6, 5, 0] = np.nan, np.inf
    out = c.run()
    assert np.isnan(out[4, 3]).all() and np.isnan(out[6, 5]).all()
    out[4, 3], out[6, 5] = clean[4, 3], clean[6, 5]
    np.testing.assert_array_equal(out.view(np.uint16), clean.view(np.uint16))


@pytest.mark.parametrize("fmt", FORMATS)
def test_equal_to_the_fp16_attention_over_the_cache_read_back(fmt):
    c = Call(62, 24, 1500, 32, 8, fmt)
    q, k, v, ks, vs, _, mask = c.tensors()
    k16, v16 = torch.empty(c.P + c.M, 8, D, dtype=torch.float16, device=DEV), torch.empty(c.P + c.M, 8, D, dtype=torch.float16, device=DEV)
    B.w4a16_kv8_read(k, v, ks, vs, fmt, 0, c.P + c.M, 8, D, k16, v16)
    want = torch.empty_like(q)
    B.tree_verify_attn(q, k16, v16, mask, want, *c.sizes(), B.new_workspace(B.tree_verify_attn_workspace_bytes(c.M, c.P, 32, 8, D)))
    torch.cuda.synchronize()
    got, want = c.run().astype(np.float64), want.cpu().numpy().astype(np.float64)
    assert np.linalg.norm(got - want) <= 2.0 ** -10 * np.linalg.norm(want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_workspace_shared_by_calls_in_a_row_and_another_stream(fmt):
    """one workspace, calls of several sizes one after another, tickets back at zero; and the same on a stream that is not the default one"""
    calls = [Call(70 + i, M, P, Hq, 8, fmt) for i, (M, P, Hq) in enumerate(((60, 900, 64), (1, 4000, 64), (24, 333, 32), (1, 5, 64)))]
    want = [c.run() for c in calls]
    ws = B.new_workspace(max(B.tree_verify_attn_kv8_workspace_bytes(c.M, c.P, c.Hq, 8, D) for c in calls))
    for c, w in zip(calls, want):
        np.testing.assert_array_equal(c.run(ws).view(np.uint16), w.view(np.uint16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c, w in zip(calls, want):
            np.testing.assert_array_equal(c.run(ws).view(np.uint16), w.view(np.uint16))


def test_graph_replays_equal_the_eager_calls():
    """append, attention and acceptance of one step captured together, replayed with other work in between"""
    M, P, Hq, Hkv, fmt = 24, 500, 32, 8, B.KV8_INT8
    rng = np.random.default_rng(5)
    qkv = dev(rng.standard_normal((M, (Hq + 2 * Hkv) * D)).astype(np.float16))
    gq, gk = dev(I.make_gamma(1, D)), dev(I.make_gamma(2, D))
    parent, _, mask = I.make_tree(3, M, 5, 3)
    token, target = I.make_verify(4, parent, p_accept=0.9)
    i32 = lambda a: dev(np.asarray(a, dtype=np.int32))
    ids = [i32(parent), i32(token), i32(target)]
    pos, maskd = dev(I.tree_positions(parent, P)), dev(mask)
    cos, sin = (dev(t) for t in I.make_rope_tables(P + 16, D))
    k0, v0 = (dev(rng.integers(0, 100, (P + M, Hkv, D), dtype=np.uint8)) for _ in range(2))
    s0 = dev((2.0 ** rng.integers(-8, -4, (P + M, Hkv))).astype(np.float16))
    k, v, ks, vs = k0.clone(), v0.clone(), s0.clone(), s0.clone()
    q, out = torch.empty(M, Hq, D, dtype=torch.float16, device=DEV), torch.empty(M, Hq, D, dtype=torch.float16, device=DEV)
    path, result = torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    ws = B.new_workspace(B.tree_verify_attn_kv8_workspace_bytes(64, 4000, 64, 8, D))

    def reset():
        k.copy_(k0), v.copy_(v0), ks.copy_(s0), vs.copy_(s0)

    def step():
        B.rope_append_kv8(qkv, gq, gk, 1e-6, pos, cos, sin, P + 16, q, k, v, ks, vs, fmt, M, P, Hq, Hkv, D)
        B.tree_verify_attn_kv8(q, k, v, ks, vs, fmt, maskd, out, M, P, Hq, Hkv, D, D ** -0.5, ws)
        B.tree_accept_kv8(*ids, M, path, result, k, v, ks, vs, P, Hkv, D)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (q, out, path, result, k, v, ks, vs)]
    graph = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(graph):
        step()
    other = Call(90, 60, 2000, 64, 8, B.KV8_E4M3)
    for replay in range(4):
        reset(), q.zero_(), out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((q, out, path, result, k, v, ks, vs), want):
            assert torch.equal(got, w), replay
        other.run(ws)


# many rows over a long prefix: taller row tiles, whose codes become fp16 numbers once for 128 rows
TALL = [
    (60, 8192, 64, 8),      # 480 rows per KV head
    (60, 16001, 64, 8),
    (64, 8191, 64, 8),      # draft keys from the last key of a step to the third step on
    (64, 6002, 64, 8),      # the last step holds two keys
    (37, 24000, 28, 4),     # 259 rows: tiles of 87
    (12, 33000, 64, 8),     # 96 rows, one tile, 31 ranges
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,P,Hq,Hkv", TALL)
def test_many_rows_over_a_long_prefix(M, P, Hq, Hkv, fmt):
    print(f"attn_kv8 tall M={M} P={P} Hq={Hq} Hkv={Hkv} fmt={fmt}", flush=True)
    c = Call(100 + M, M, P, Hq, Hkv, fmt, tree="random", q_std=3.0)
    out = c.run()
    c.check(out)
    np.testing.assert_array_equal(c.run().view(np.uint16), out.view(np.uint16))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("at", [5, 8190, 8230])
def test_nan_keys_and_values_under_many_rows(at, fmt):
    """as above: a NaN scale reaches the rows that see its key, and only the heads of its KV head"""
    c = Call(110 + at, 60, 8190, 64, 8, fmt, tree="random")
    c.ks[at, 3], c.k[at, 3] = np.nan, 0
    c.vs[at, 5], c.v[at, 5] = np.nan, 0
    out = c.run()
    c.check(out)
    lost = np.isnan(out).any(axis=(0, 2))
    assert lost[24:32].all() and lost[40:48].all() and lost.sum() == 16


@pytest.mark.parametrize("fmt", FORMATS)
def test_hidden_rows_that_hold_anything_under_many_rows(fmt):
    M, P = 64, 9001
    c = Call(120, M, P, 64, 8, fmt)
    n = 41
    c.mask[n:], c.mask[:, n:] = 0, 0
    clean = c.run()
    c.check(clean)
    rng = np.random.default_rng(M)
    for codes, scales in ((c.k, c.ks), (c.v, c.vs)):
        codes[P + n:] = rng.choice(np.array([0x7F, 0xFF, 0x80, 0x7E], dtype=np.uint8), codes[P + n:].shape)
        scales[P + n:] = rng.choice(np.array([np.nan, np.inf, -np.inf, 65504.0, 1.0], dtype=np.float16), scales[P + n:].shape)
    np.testing.assert_array_equal(c.run().view(np.uint16), clean.view(np.uint16))


def test_workspace_shared_by_calls_of_every_kind():
    """few and many rows, short and long prefixes, one workspace, one after another, twice"""
    calls = [Call(130 + i, *c) for i, c in enumerate(((60, 8192, 64, 8, 1), (1, 2048, 64, 8, 2), (7, 40000, 32, 8, 1), (60, 700, 64, 8, 2), (12, 33000, 64, 8, 1)))]
    want = [c.run() for c in calls]
    ws = B.new_workspace(max(B.tree_verify_attn_kv8_workspace_bytes(c.M, c.P, c.Hq, c.Hkv, D) for c in calls))
    for _ in range(2):
        for c, w in zip(calls, want):
            np.testing.assert_array_equal(c.run(ws).view(np.uint16), w.view(np.uint16))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,P,Hq,Hkv", [(5, 40, 8, 2), (37, 3333, 28, 4), (60, 8190, 64, 8)])
def test_rows_of_padding_are_zero_whatever_the_prefix_holds(M, P, Hq, Hkv, fmt):
    """an empty mask row sees no committed key either: neither a NaN key there nor a NaN or an infinity in the row's own query shows"""
    c = Call(140 + M, M, P, Hq, Hkv, fmt)
    c.mask[M - 2:], c.mask[:, M - 2:] = 0, 0
    c.mask[1] = 0     # and one inside the tree
    out = c.run()
    c.check(out)
    c.ks[3, 1], c.k[3, 1] = np.nan, 0
    c.q[1, 0], c.q[M - 1, 0, 5], c.q[M - 2, 0, 5] = np.inf, np.nan, -np.inf
    out = c.run()
    assert (out[[1, M - 2, M - 1]] == 0).all() and np.isnan(out[0]).any()


def test_nan_keys_and_hidden_rows_under_many_rows_of_e4m3():
    """as the three above in one, over a prefix that makes the tall tiles worth it for e4m3 as well"""
    M, P, n = 60, 16001, 44
    c = Call(150, M, P, 64, 8, B.KV8_E4M3, tree="random")
    c.mask[n:], c.mask[:, n:] = 0, 0
    for at, head in ((7, 3), (P + 20, 5)):
        c.ks[at, head], c.k[at, head] = np.nan, 0
    out = c.run()
    c.check(out)
    lost = np.isnan(out[:n]).any(axis=(0, 2))
    assert lost[24:32].all() and lost[40:48].all() and lost.sum() == 16 and (out[n:] == 0).all()
    rng = np.random.default_rng(M)
    for codes, scales in ((c.k, c.ks), (c.v, c.vs)):
        codes[P + n:] = rng.choice(np.array([0x7F, 0xFF, 0x80, 0x7E], dtype=np.uint8), codes[P + n:].shape)
        scales[P + n:] = rng.choice(np.array([np.nan, np.inf, -np.inf, 65504.0, 1.0], dtype=np.float16), scales[P + n:].shape)
    np.testing.assert_array_equal(c.run().view(np.uint16), out.view(np.uint16))


@pytest.mark.parametrize("M,Hq", [(3, 64), (16, 512)])   # one row tile per KV head, and tiles of 128 rows
def test_a_cache_of_more_than_4_gib(M, Hq):
    """P = 560000 rows of 64 heads: 4.6 GB of K codes and as much of V.  All keys are zero but a few, on both sides of the 4 GiB boundary, and the draft's:
    append, read, attention, acceptance."""
    P, Hkv, fmt = 560000, 64, B.KV8_INT8
    print(f"attn_kv8 long cache M={M} Hq={Hq}", flush=True)
    T, edge = P + M, 2 ** 32 // (Hkv * D)
    rng = np.random.default_rng(M)
    k, v = (torch.zeros(T, Hkv, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.ones(T, Hkv, dtype=torch.float16, device=DEV) for _ in range(2))
    at = np.array([0, 1, edge - 1, edge, edge + 1, P - 1])
    small = Call(160, 1, len(at) - 1, Hkv, Hkv, fmt)
    for big, part in ((k, small.k), (v, small.v), (ks, small.ks * np.float16(3)), (vs, small.vs)):
        big[torch.from_numpy(at).to(DEV)] = dev(part)
    qkv = (rng.standard_normal((M, (Hq + 2 * Hkv) * D)) * 2).astype(np.float16)
    pos, (cos, sin) = np.arange(M, dtype=np.int32), I.make_rope_tables(M, D)
    q = torch.empty(M, Hq, D, dtype=torch.float16, device=DEV)
    B.rope_append_kv8(dev(qkv), None, None, 0.0, dev(pos), dev(cos), dev(sin), M, q, k, v, ks, vs, fmt, M, P, Hq, Hkv, D)
    draft = qkv.reshape(M, -1, D)[:, Hq + Hkv:]
    codes, scales = R.kv8_quantise(draft, fmt)
    np.testing.assert_array_equal(v[P:].cpu().numpy(), codes)
    np.testing.assert_array_equal(vs[P:].cpu().numpy(), scales)
    # read: the last rows
    rows = P + M - (edge - 2)
    k16, v16 = torch.empty(rows, Hkv, D, dtype=torch.float16, device=DEV), torch.empty(rows, Hkv, D, dtype=torch.float16, device=DEV)
    B.w4a16_kv8_read(k, v, ks, vs, fmt, edge - 2, rows, Hkv, D, k16, v16)
    seen = np.concatenate([at, P + np.arange(M)])
    take = lambda t: t[torch.from_numpy(seen).to(DEV)].cpu().numpy()
    kk, vv = R.kv8_values(take(k), take(ks), fmt), R.kv8_values(take(v), take(vs), fmt)
    late = seen >= edge - 2
    np.testing.assert_array_equal(k16[torch.from_numpy(seen[late] - (edge - 2)).to(DEV)].cpu().numpy(), kk[late].astype(np.float16))
    np.testing.assert_array_equal(v16[torch.from_numpy(seen[late] - (edge - 2)).to(DEV)].cpu().numpy(), vv[late].astype(np.float16))
    assert not (k16[0].any() or v16[0].any())
    del k16, v16
    # attention: a row sees the committed rows -- P - 6 of them zeros -- and the draft up to itself
    mask = I.chain_tree(M)[2]
    out = torch.empty(M, Hq, D, dtype=torch.float16, device=DEV)
    B.tree_verify_attn_kv8(q, k, v, ks, vs, fmt, dev(mask), out, M, P, Hq, Hkv, D, D ** -0.5, B.new_workspace(B.tree_verify_attn_kv8_workspace_bytes(M, P, Hq, Hkv, D)))
    out, qh = out.cpu().numpy().astype(np.float64), q.cpu().numpy().astype(np.float64)
    rep, reach = Hq // Hkv, 0
    for i in range(M):
        for head in range(0, Hq, max(1, Hq // 16) + 1):
            g = head // rep
            visible = np.concatenate([np.ones(len(at), dtype=bool), mask[i] != 0])
            s = (kk[visible, g] @ qh[i, head]) * D ** -0.5
            m = max(s.max(), 0.0)
            w = np.exp(s - m)
            den = w.sum() + (P - len(at)) * np.exp(-m)
            want, spread = (w / den) @ vv[visible, g], (w / den) @ np.abs(vv[visible, g])
            qk = np.abs(qh[i, head]).sum() * np.abs(kk[visible, g]).max() * D ** -0.5
            # as at the top; a zero key's probability of exp(-m), 2^-11 of it off in the sum as well
            tol = spread * (2 * 2.0 ** -11 * 1.01 + 2 * 128 * 2.0 ** -24 * min(qk, 64.0 * 8)) + np.abs(want) * 2.0 ** -11 + 2.0 ** -25 + T * 2.0 ** -25 * np.abs(vv[visible, g]).max() / T ** 0.5
            assert (np.abs(out[i, head] - want) <= tol).all(), (i, head, np.abs(out[i, head] - want).max(), tol.min())
            reach += np.abs(want).max() > 0.05
    assert reach > M   # the planted rows do show
    # acceptance moves rows beyond the boundary
    parent, token = np.array([-1, 0, 0] + [2] * (M - 3), dtype=np.int32), np.arange(M, dtype=np.int32)
    target = np.array([2] + [M + 5] * (M - 1), dtype=np.int32)
    path, result = torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    third = [t[P + 2].clone() for t in (k, v, ks, vs)]
    B.tree_accept_kv8(dev(parent), dev(token), dev(target), M, path, result, k, v, ks, vs, P, Hkv, D)
    assert result.tolist() == [2, M + 5] and all(torch.equal(t[P + 1], w) for t, w in zip((k, v, ks, vs), third))


STRANGE = {   # (format, code, scale): values that no append writes -- no number, or beyond fp16
    "nan": (B.KV8_E4M3, 0x7F, 0.25),
    "minus_nan_zero_scale": (B.KV8_E4M3, 0xFF, np.nan),
    "e4m3_beyond_fp16": (B.KV8_E4M3, 0x7E, 256.0),
    "int8_beyond_fp16": (B.KV8_INT8, 0x80, 512.0),
    "int8_infinite": (B.KV8_INT8, 0x7F, np.inf),
}


@pytest.mark.parametrize("strange", list(STRANGE))
@pytest.mark.parametrize("M,P,Hq,Hkv", [(12, 96, 8, 2), (33, 31, 8, 1), (64, 1000, 28, 4), (60, 16001, 64, 8)])
def test_codes_that_are_no_numbers_stay_with_the_rows_that_see_them(M, P, Hq, Hkv, strange):
    """a draft key that some rows see and others do not: what it holds reaches the rows that see it, of its KV head, and leaves the others' bits alone"""
    fmt, code, scale = STRANGE[strange]
    print(f"attn_kv8 strange codes M={M} P={P} Hq={Hq} Hkv={Hkv} {strange}", flush=True)
    c = Call(170 + M, M, P, Hq, Hkv, fmt, tree="random")
    clean = c.run()
    c.check(clean)
    seen_by = c.mask.sum(0)
    node = int(np.flatnonzero((seen_by > 1) & (seen_by < M))[-1])
    sees, kvh = c.mask[:, node] != 0, Hkv - 1
    heads = slice(kvh * (Hq // Hkv), Hq)
    for which in "kv":
        d = Call(170 + M, M, P, Hq, Hkv, fmt, tree="random")
        getattr(d, which)[P + node, kvh, 77] = code
        getattr(d, which + "s")[P + node, kvh] = scale
        out = d.run()
        same = np.ones((M, Hq), dtype=bool)
        same[sees, heads] = False
        np.testing.assert_array_equal(out[same].view(np.uint16), clean[same].view(np.uint16))
        if which == "v":
            assert not np.isfinite(out[sees, heads, 77].astype(np.float64)).any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,P,Hq,Hkv", [(1, 0, 8, 2), (3, 300, 8, 2), (40, 5000, 64, 8), (60, 16001, 64, 8)])
def test_scores_that_are_all_minus_infinity_are_nan(M, P, Hq, Hkv, fmt):
    """a row's weights are then 0 / 0, as in tree_verify_attn: by one range, by several and by either merge"""
    c = Call(180 + M, M, P, Hq, Hkv, fmt)
    c.k[:, :, 9] = 1 if fmt == B.KV8_INT8 else 0x38      # one: positive in every key
    clean = c.run()
    c.q[M - 1, 2, 9] = -np.inf
    out = c.run()
    assert np.isnan(out[M - 1, 2]).all()
    out[M - 1, 2] = clean[M - 1, 2]
    np.testing.assert_array_equal(out.view(np.uint16), clean.view(np.uint16))


PLANS = [   # M, P, Hq, Hkv, formats, what the call's plan has to be: rows of a tile, tiles per KV head, ranges, last workgroup merges, tiles of up to 128 rows
    (1, 700, 64, 8, FORMATS, (8, 1, None, 1, 0)),            # tiles of 32 rows: merged by their last workgroup,
    (12, 33000, 64, 8, [B.KV8_E4M3], (32, 3, 10, 0, 0)),     # by a second kernel,
    (64, 100, 64, 64, FORMATS, (32, 2, 1, 0, 0)),            # one range
    (5, 77, 1024, 1024, FORMATS, (5, 1, 1, 0, 0)),           # 1024 workgroups
    (64, 8191, 64, 8, FORMATS, (128, 4, 8, 0, 1)),           # tiles of 128 rows
    (37, 24000, 28, 4, [B.KV8_INT8], (87, 3, 21, 0, 1)),
    (12, 64000, 64, 8, [B.KV8_E4M3], (96, 1, 32, 0, 1)),
    (64, 500, 512, 64, FORMATS, (128, 4, 1, 0, 1)),          # one range: 256 workgroups
    (33, 40, 1024, 128, FORMATS, (88, 3, 1, 0, 1)),          # 384
    (8, 300, 4096, 512, FORMATS, (64, 1, 1, 0, 1)),          # 512
    (64, 0, 512, 64, FORMATS, (128, 4, 1, 0, 1)),
]


@pytest.mark.parametrize("M,P,Hq,Hkv,fmt,plan", [(*c[:4], fmt, c[5]) for c in PLANS for fmt in c[4]])
def test_every_kind_of_plan(M, P, Hq, Hkv, fmt, plan):
    """parity, rows of padding, hidden rows that hold anything and NaN keys, with the kernel and the merge that run known"""
    print(f"attn_kv8 plan M={M} P={P} Hq={Hq} Hkv={Hkv} fmt={fmt}", flush=True)
    got = B.tree_verify_attn_kv8_plan_describe(M, P, Hq, Hkv, D, fmt)
    assert all(w is None or g == w for g, w in zip(got, plan)), got
    c = Call(190 + M + P, M, P, Hq, Hkv, fmt)
    n = M - M // 4
    c.mask[n:], c.mask[:, n:] = 0, 0
    clean = c.run()
    c.check(clean)
    assert (clean[n:] == 0).all()
    rng = np.random.default_rng(M)
    for codes, scales in ((c.k, c.ks), (c.v, c.vs)):
        codes[P + n:] = rng.choice(np.array([0x7F, 0xFF, 0x80, 0x7E], dtype=np.uint8), codes[P + n:].shape)
        scales[P + n:] = rng.choice(np.array([np.nan, np.inf, -np.inf, 65504.0, 1.0], dtype=np.float16), scales[P + n:].shape)
    np.testing.assert_array_equal(c.run().view(np.uint16), clean.view(np.uint16))
    if M > 1:   # a draft key that not every node sees
        node, group = int(np.argmin(c.mask[:n, :n].sum(0))), Hq // Hkv
        c.vs[P + node, 0], c.v[P + node, 0] = np.nan, 0
        out, sees = c.run(), c.mask[:, node] != 0
        assert np.isnan(out[sees, :group]).all()
        out[sees, :group] = clean[sees, :group]
        np.testing.assert_array_equal(out.view(np.uint16), clean.view(np.uint16))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,P,Hq,Hkv,tall", [(1, 6000, 8, 8, 0), (16, 6000, 128, 128, 0), (60, 16001, 64, 8, 1), (16, 6000, 1032, 129, 1)])
def test_probabilities_below_the_normal_range_of_fp16_count(M, P, Hq, Hkv, tall, fmt):
    """One committed key scores 15.5 binary orders above all others, which weigh w = 2^-15.5 each: its value is 0, theirs is 1, so an output is n w / (1 + n w).
    Each w is rounded by at most 2^-25."""
    assert B.tree_verify_attn_kv8_plan_describe(M, P, Hq, Hkv, D, fmt)[4] == tall
    print(f"attn_kv8 small probabilities M={M} P={P} Hq={Hq} Hkv={Hkv} fmt={fmt}", flush=True)
    one = 1 if fmt == B.KV8_INT8 else 0x38
    T = P + M
    k, v = torch.zeros(T, Hkv, D, dtype=torch.uint8, device=DEV), torch.full((T, Hkv, D), one, dtype=torch.uint8, device=DEV)
    ks, vs = torch.ones(T, Hkv, dtype=torch.float16, device=DEV), torch.ones(T, Hkv, dtype=torch.float16, device=DEV)
    q, out = torch.zeros(M, Hq, D, dtype=torch.float16, device=DEV), torch.empty(M, Hq, D, dtype=torch.float16, device=DEV)
    q[:, :, 5] = 64.0
    scale = 15.5 * np.log(2.0) / 64.0
    mask, ws = dev(np.tril(np.ones((M, M), dtype=np.uint8))), B.new_workspace(B.tree_verify_attn_kv8_workspace_bytes(M, P, Hq, Hkv, D))
    for at in (0, 31, P // 2, P - 1):
        k[at, :, 5], v[at] = one, 0
        B.tree_verify_attn_kv8(q, k, v, ks, vs, fmt, mask, out, M, P, Hq, Hkv, D, scale, ws)
        torch.cuda.synchronize()
        k[at, :, 5], v[at] = 0, one
        n = P + np.arange(M)[:, None, None]      # others than `at` that row i sees
        w = 2.0 ** -15.5
        want = n * w / (1 + n * w)
        # a weight's rounding, the scores' (15.5 in fp32, a few steps of 2^-20) and the output's
        tol = n * 2.0 ** -25 + want * (2.0 ** -11 + 2.0 ** -17)
        err = np.abs(out.cpu().numpy().astype(np.float64) - want)
        assert (err <= tol).all(), (at, (err / tol).max())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,P,Hq,Hkv", [(9, 700, 16, 4), (60, 16001, 64, 8)])
def test_values_and_keys_below_the_normal_range_of_fp16(M, P, Hq, Hkv, fmt):
    """scales at the formats' lower end: every value, then every key, is a subnormal fp16 number"""
    c = Call(200 + M, M, P, Hq, Hkv, fmt)
    rng = np.random.default_rng(M)
    if fmt == B.KV8_INT8:
        least = lambda codes: (codes, (rng.integers(1, 4, (P + M, Hkv)) * 2.0 ** -24).astype(np.float16))
    else:   # codes of up to 1.875 times 2^-15
        least = lambda codes: ((codes & 0x80) | rng.integers(1, 0x40, codes.shape).astype(np.uint8), np.full((P + M, Hkv), 2.0 ** -15, dtype=np.float16))
    v, vs = c.v, c.vs
    c.v, c.vs = least(c.v)
    out = c.run()
    k64, v64 = R.kv8_values(c.k, c.ks, fmt), R.kv8_values(c.v, c.vs, fmt)
    assert np.abs(v64).max() < 2.0 ** -14
    want, spread = R.tree_verify_attn_seen(c.q, k64, v64, c.mask, c.scale)
    qk = np.abs(c.q.astype(np.float64)).sum(-1).max() * np.abs(k64).max() * c.scale      # above every sum |q k| scale
    tol = spread * (2.0 ** -11 * 1.01 + 2 * 128 * 2.0 ** -24 * qk) + (P + M) * 2.0 ** -25 * np.abs(v64).max() + 2.0 ** -25 * 1.01   # the output is a multiple of 2^-24
    assert (np.abs(out.astype(np.float64) - want) <= tol).all()
    c.v, c.vs = v, vs
    c.k, c.ks = least(c.k)
    c.q = (c.q.astype(np.float32) * 2000).astype(np.float16)
    assert np.abs(R.kv8_values(c.k, c.ks, fmt)).max() < 2.0 ** -14
    c.check(c.run())
