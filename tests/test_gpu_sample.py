"""GPU: lm_head_sample through the C ABI against the oracle.  Tokens have to be equal wherever the oracle's margin -- the distance of u, top_p or
min_p from the nearest border -- exceeds what the definition leaves open: weights are rounded to 2^-44 and tokens beyond e^-31 dropped, together
below V (2^-45 + e^-31) of the row's weight; the probability is fp32."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
NONE = 0x7FFFFFFF


def run(logits, temperature=None, top_k=None, top_p=None, min_p=None, u=0.0, ws=None):
    logits = torch.as_tensor(logits, dtype=torch.float32)
    M, V = logits.shape
    f = lambda t, dtype=torch.float32: None if t is None else torch.as_tensor(np.broadcast_to(t, (M,)).copy(), dtype=dtype).to(DEV)
    token = torch.full((M + 1,), 777, dtype=torch.int32, device=DEV)
    prob = torch.full((M + 1,), 7.0, dtype=torch.float32, device=DEV)
    ws = B.new_workspace(B.lm_head_sample_workspace_bytes(M, V)) if ws is None else ws
    B.lm_head_sample(logits.to(DEV), M, V, f(temperature), f(top_k, torch.int32), f(top_p), f(min_p), f(u), token, prob, ws)
    torch.cuda.synchronize()
    assert int(token[M]) == 777 and float(prob[M]) == 7
    return token[:M].cpu().numpy(), prob[:M].cpu().numpy()


def check(logits, temperature=None, top_k=None, top_p=None, min_p=None, u=0.0, ws=None):
    token, prob = run(logits, temperature, top_k, top_p, min_p, u, ws)
    x = torch.as_tensor(logits, dtype=torch.float32).numpy()
    M, V = x.shape
    f32 = lambda t, d: np.broadcast_to(np.asarray(d if t is None else t, dtype=np.float32), (M,)).astype(np.float64)
    T, P, Q, U = f32(temperature, 1), f32(top_p, 1), f32(min_p, 0), f32(u, 0)
    K = np.broadcast_to(np.asarray(0 if top_k is None else top_k), (M,))
    close = 0
    for m in range(M):
        want, p, margin = R.sample(x[m], T[m], int(K[m]), P[m], Q[m], U[m])
        if margin == 0 or margin > V * (2.0 ** -45 + 3.5e-14):   # 0: equal weights, whose sums are exact on either side, and the border itself
            assert token[m] == want, (m, token[m], want, margin)
            assert abs(prob[m] - p) <= 2.0 ** -23 * p + V * 6.5e-14 * p, (m, prob[m], p)
        else:
            close += 1
    assert close <= max(1, M // 20)
    return token, prob


def rows(seed, M, V, std=2.2):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((M, V)) * std + 12 * rng.random((M, V)) ** 200).astype(np.float32), rng


LIMITS = ["none", "k", "p", "min", "kp", "kmin", "pmin", "all"]


@pytest.mark.parametrize("limits", LIMITS)
@pytest.mark.parametrize("M,V", [(1, 1), (3, 2), (2, 63), (64, 100), (5, 1025), (4, 4099), (2, 8193), (3, 32000), (1, 128256)])
def test_random_rows(M, V, limits):
    print(f"sample M={M} V={V} {limits}", flush=True)
    x, rng = rows(V + M, M, V)
    full = limits == "all"
    k = rng.integers(1, min(V, 300) + 1, M) if "k" in limits or full else None
    p = rng.uniform(0.5, 1.0, M) if limits in ("p", "kp", "pmin") or full else None
    q = rng.uniform(0.0, 0.2, M) if "min" in limits or full else None
    check(x, rng.uniform(0.4, 1.6, M), k, p, q, rng.random(M))


@pytest.mark.parametrize("V", [1000, 40000])
@pytest.mark.parametrize("temperature", [0.02, 1.0, 7.0, 300.0, 1e30, float("inf")])
def test_temperatures(V, temperature):
    """from nearly greedy to uniform: at high temperatures thousands of tokens have nearly the same weight"""
    x, rng = rows(3, 6, V)
    for limits in (dict(), dict(top_p=0.9), dict(top_k=V // 3), dict(top_k=V // 2, top_p=0.7, min_p=0.05)):
        check(x, temperature, u=rng.random(6), **limits)


@pytest.mark.parametrize("V", [5, 3000, 20000])
def test_equal_logits_stay_in_token_order(V):
    """all weights 1 or two levels: every border falls between equal logits"""
    x = np.zeros((4, V), dtype=np.float32)
    x[1, ::2] = -0.0
    x[2, V // 3:] = np.log(0.5)
    x[3, :V // 2] = -1.0
    u = np.array([0.0, 0.37, 0.999, 0.61])
    for limits in (dict(), dict(top_k=max(1, V // 4)), dict(top_p=0.61803), dict(top_k=max(1, V - 2), top_p=0.3333), dict(min_p=0.6), dict(top_k=max(2, V // 2 + 1), min_p=0.4)):
        check(x, None, u=u, **limits)


def test_greedy_rows_and_limits_out_of_range():
    x, rng = rows(8, 8, 5000)
    x[:, 4000] = x[:, 1234] = 40.0
    u = rng.random(8)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=nan), dict(top_k=1), dict(top_p=0.0), dict(top_p=-3.0), dict(min_p=1.5), dict(min_p=inf)):
        token, prob = run(x, u=u, **kw)
        assert (token == 1234).all() and (prob == 1).all(), kw
    plain = run(x, u=u)
    for kw in (dict(top_k=0), dict(top_k=-5), dict(top_k=5000), dict(top_k=2 ** 31 - 1), dict(top_p=1.0), dict(top_p=9.0), dict(top_p=nan), dict(min_p=0.0), dict(min_p=-1.0),
               dict(min_p=nan), dict(temperature=1.0)):
        token, prob = run(x, u=u, **kw)
        assert (token == plain[0]).all() and (prob == plain[1]).all(), kw
    for low, high in ((-1.0, 0.0), (nan, 0.0), (1.0, 1 - 2.0 ** -24), (5.0, 1 - 2.0 ** -24), (inf, 1 - 2.0 ** -24)):
        assert (run(x, 2.0, u=low)[0] == run(x, 2.0, u=high)[0]).all()


def test_banned_tokens_infinities_nan_and_empty_rows():
    x, rng = rows(9, 9, 9001)
    inf, nan = np.inf, np.nan
    x[0, rng.random(9001) < 0.5] = -inf
    x[1] = -inf
    x[2] = nan
    x[3], x[3, 77] = -inf, -5.0
    x[4, 10], x[4, 9000] = inf, inf
    x[5, ::3] = nan
    x[6, rng.random(9001) < 0.9] = np.finfo(np.float32).min     # the type's lowest value as a mask
    x[7] = np.finfo(np.float32).min
    x[8], x[8, 5] = np.finfo(np.float32).max, -np.finfo(np.float32).max
    for limits in (dict(), dict(top_k=40), dict(top_p=0.8), dict(top_k=5000, top_p=0.9, min_p=0.01)):
        for u in (0.0, 0.5, 1 - 2.0 ** -24):
            token, prob = check(x, 1.3, u=u, **limits)
            assert token[1] == token[2] == NONE and prob[1] == prob[2] == 0
            assert token[3] == 77 and prob[3] == 1 and token[4] in (10, 9000)
    assert run(x, 0.0)[0][1] == NONE


def test_last_tokens_of_a_row_and_the_largest_vocabulary():
    for V in (262144, 131071, 8192, 8191, 1024):
        x = np.full((2, V), -3.0, dtype=np.float32)
        x[0, V - 1], x[1, V - 2] = 9.0, 9.0
        token, _ = run(x, 0.5, u=[0.5, 0.5])
        assert list(token) == [V - 1, V - 2]
        check(x, 3.0, top_p=0.9, u=[1 - 2.0 ** -24, 0.99])


def test_frequencies():
    """a stratified grid of u draws every token as often as its share says, within one"""
    x, _ = rows(10, 1, 37)
    p = np.exp(x[0].astype(np.float64) - x[0].max())
    p /= p.sum()
    counts = np.zeros(37)
    for i in range(32):
        u = (np.arange(64) + 64 * i + 0.5) / 2048
        token, _ = run(np.repeat(x, 64, 0), u=u)
        counts += np.bincount(token, minlength=37)
    assert (np.abs(counts - p * 2048) <= 1).all()


def test_rows_do_not_depend_on_their_neighbours_or_on_the_call():
    x, rng = rows(11, 64, 20011)
    kw = dict(temperature=rng.uniform(0.5, 2, 64), top_k=rng.integers(1, 5000, 64), top_p=rng.uniform(0.5, 1, 64), min_p=rng.uniform(0, 0.1, 64), u=rng.random(64))
    ws = B.new_workspace(B.lm_head_sample_workspace_bytes(64, 262144))
    token, prob = run(x, ws=ws, **kw)
    again = run(x, ws=ws, **kw)
    assert (again[0] == token).all() and (again[1] == prob).all()
    for m in (0, 13, 63):
        one = run(x[m:m + 1], ws=ws, **{n: v[m:m + 1] for n, v in kw.items()})
        assert one[0][0] == token[m] and one[1][0] == prob[m]


@pytest.mark.parametrize("V", [128256, 262144])
def test_rows_do_not_depend_on_how_many_there_are(V):
    """64 long rows are split into fewer, longer pieces than one is"""
    x, rng = rows(14, 64, V)
    kw = dict(temperature=rng.uniform(0.5, 1.5, 64), top_k=rng.integers(-5, 3000, 64), top_p=rng.uniform(0.5, 1.1, 64), min_p=rng.uniform(-0.1, 0.01, 64), u=rng.random(64))
    token, prob = run(x, **kw)
    for m in range(0, 64, 9):
        one = run(x[m:m + 1], **{n: v[m:m + 1] for n, v in kw.items()})
        assert one[0][0] == token[m] and one[1][0] == prob[m]


def test_equal_logits_in_the_largest_call():
    """a whole row in one bin: the first k tokens stay, or the first ceil(p V); token j of n equal ones is drawn for u in [j / n, (j + 1) / n)"""
    V, rng = 262144, np.random.default_rng(15)
    x = np.zeros((64, V), dtype=np.float32)
    u = rng.integers(0, 1 << 24, 64).astype(np.float64) / (1 << 24)
    k = rng.integers(2, V, 64)
    token, prob = run(x, top_k=k, u=u)
    np.testing.assert_array_equal(token, np.floor(u * k).astype(np.int64))
    np.testing.assert_array_equal(prob, (1.0 / k).astype(np.float32))
    p = rng.integers(1, 256, 64) / 256.0
    n = np.ceil(p * V)
    token, prob = run(x, top_p=p, u=u)
    np.testing.assert_array_equal(token, np.floor(u * n).astype(np.int64))
    np.testing.assert_array_equal(prob, (1.0 / n).astype(np.float32))


def test_graph_replays_and_another_stream():
    x, rng = rows(12, 5, 50000)
    d = lambda a, t=torch.float32: torch.as_tensor(np.asarray(a), dtype=t).to(DEV)
    logits, T, k, p = d(x), d(rng.uniform(0.5, 1.5, 5)), d(rng.integers(1, 400, 5), torch.int32), d(rng.uniform(0.6, 1, 5))
    u, token, prob = torch.zeros(5, device=DEV), torch.empty(5, dtype=torch.int32, device=DEV), torch.empty(5, device=DEV)
    ws = B.new_workspace(B.lm_head_sample_workspace_bytes(5, 50000))
    call = lambda: B.lm_head_sample(logits, 5, 50000, T, k, p, None, u, token, prob, ws)
    draws = [d(rng.random(5)) for _ in range(4)]
    wants = []
    for r in draws:
        u.copy_(r)
        call()
        torch.cuda.synchronize()
        wants.append((token.clone(), prob.clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for r, want in zip(draws, wants):
        u.copy_(r), token.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, want[0]) and torch.equal(prob, want[1])
        run(x[:2], 1.0, top_p=0.5, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        side.synchronize()
    assert torch.equal(token, wants[-1][0])


def test_one_step_from_the_projection_to_the_token():
    """the operators together: norms, rotation, 8-bit cache, attention, LM head, sampled token"""
    M, P, Hq, Hkv, D, V, fmt = 6, 200, 16, 4, 128, 1500, B.KV8_INT8
    gen = torch.Generator(device=DEV).manual_seed(3)
    half = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device=DEV) * std).half()
    empty = lambda *s, dtype=torch.float16: torch.empty(*s, dtype=dtype, device=DEV)
    from paper_2505_22179_amd import inputs as I
    cos, sin = (torch.from_numpy(t).to(DEV) for t in I.make_rope_tables(P + 16, D))
    mask = torch.from_numpy(I.chain_tree(M)[2]).to(DEV)
    gq, gk = 1 + half(D, std=0.1), 1 + half(D, std=0.1)
    k, v = torch.zeros(P + M, Hkv, D, dtype=torch.int8, device=DEV), torch.zeros(P + M, Hkv, D, dtype=torch.int8, device=DEV)
    ks, vs = empty(P + M, Hkv), empty(P + M, Hkv)
    prompt, qkv = half(P, (Hq + 2 * Hkv) * D), half(M, (Hq + 2 * Hkv) * D)
    q, qp, out = empty(M, Hq, D), empty(P, Hq, D), empty(M, Hq, D)
    i32 = lambda lo, hi: torch.arange(lo, hi, dtype=torch.int32, device=DEV)
    B.rope_append_kv8(prompt, gq, gk, 1e-6, i32(0, P), cos, sin, P + 16, qp, k, v, ks, vs, fmt, P, 0, Hq, Hkv, D)
    B.rope_append_kv8(qkv, gq, gk, 1e-6, i32(P, P + M), cos, sin, P + 16, q, k, v, ks, vs, fmt, M, P, Hq, Hkv, D)
    B.tree_verify_attn_kv8(q, k, v, ks, vs, fmt, mask, out, M, P, Hq, Hkv, D, D ** -0.5, B.new_workspace(B.tree_verify_attn_kv8_workspace_bytes(M, P, Hq, Hkv, D)))
    W = half(V, Hq * D, std=0.05)
    packed = empty(B.lm_head_packed_bytes(V, Hq * D), dtype=torch.uint8)
    B.lm_head_pack(W, packed, V, Hq * D)
    logits, idx, lp = empty(M, V, dtype=torch.float32), empty(M, 4, dtype=torch.int32), empty(M, 4, dtype=torch.float32)
    B.lm_head_topk(out, packed, M, V, Hq * D, 4, logits, idx, lp, empty(B.lm_head_workspace_bytes(M, V, Hq * D, 4), dtype=torch.uint8))
    T, u = torch.full((M,), 0.8, device=DEV), torch.rand(M, generator=gen, device=DEV)
    topk = torch.full((M,), 50, dtype=torch.int32, device=DEV)
    token, prob = empty(M, dtype=torch.int32), empty(M, dtype=torch.float32)
    B.lm_head_sample(logits, M, V, T, topk, None, None, u, token, prob, B.new_workspace(B.lm_head_sample_workspace_bytes(M, V)))
    torch.cuda.synchronize()
    # the same in 64 bits: attention over exact keys and values differs by the cache's rounding, so it is held to that of the stored ones
    allqkv, c = torch.cat([prompt, qkv]).cpu().numpy(), np.zeros((P + M, Hkv, D), dtype=np.float16)
    q64, k64, v64 = R.rope_append_qk_norm(allqkv, gq.cpu().numpy(), gk.cpu().numpy(), 1e-6, np.arange(P + M), cos.cpu().numpy(), sin.cpu().numpy(), c, c, 0, Hq, Hkv, D)
    stored = [R.kv8_values(*R.kv8_quantise(t.astype(np.float16), fmt), fmt) for t in (k64, v64)]
    want, _ = R.tree_verify_attn_seen(q64[P:], *stored, mask.cpu().numpy(), D ** -0.5)
    got = out.cpu().numpy().astype(np.float64)
    assert np.linalg.norm(got - want) <= 2e-3 * np.linalg.norm(want)
    x = logits.cpu().numpy()
    exact = got.reshape(M, -1) @ W.cpu().numpy().astype(np.float64).T
    assert np.abs(x - exact).max() <= 1e-3
    for m in range(M):
        t, p, margin = R.sample(x[m], float(np.float32(0.8)), 50, 1.0, 0.0, float(u[m]))
        assert margin < 1e-9 or (int(token[m]) == t and abs(float(prob[m]) - p) <= 1e-6 * p)


def test_two_graphs_that_share_a_workspace():
    """attention and sampling of two steps of different sizes, captured apart, replayed in turn with eager calls in between, all on one workspace"""
    rng = np.random.default_rng(21)
    d = lambda a, t=torch.float32: torch.as_tensor(np.asarray(a), dtype=t).to(DEV)
    D, fmt, V = 128, B.KV8_INT8, 40000
    steps = []
    ws = B.new_workspace(max(B.tree_verify_attn_kv8_workspace_bytes(60, 9000, 64, 8, D), B.lm_head_sample_workspace_bytes(60, V)))
    for M, P, Hq, Hkv in ((60, 9000, 64, 8), (3, 1500, 32, 8)):
        x, _ = rows(30 + M, M, V)
        codes = [d(rng.integers(0, 256, (P + M, Hkv, D)), torch.uint8) for _ in range(2)]
        scales = [d(rng.integers(8, 16, (P + M, Hkv)) / 2048.0, torch.float16) for _ in range(2)]
        q, out = d(rng.standard_normal((M, Hq, D)), torch.float16), torch.empty(M, Hq, D, dtype=torch.float16, device=DEV)
        args = d(x), M, V, d(rng.uniform(0.5, 1.5, M)), d(rng.integers(1, 400, M), torch.int32), d(rng.uniform(0.6, 1, M)), None, d(rng.random(M))
        token, prob, mask = torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(M, device=DEV), torch.tril(torch.ones(M, M, dtype=torch.uint8, device=DEV))

        def step(q=q, codes=codes, scales=scales, mask=mask, out=out, M=M, P=P, Hq=Hq, Hkv=Hkv, args=args, token=token, prob=prob):
            B.tree_verify_attn_kv8(q, *codes, *scales, fmt, mask, out, M, P, Hq, Hkv, D, D ** -0.5, ws)
            B.lm_head_sample(*args, token, prob, ws)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        steps.append((step, graph, (out, token, prob), [t.clone() for t in (out, token, prob)]))
    for turn in range(3):
        for step, graph, got, want in steps:
            for t in got:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
        steps[turn % 2][0]()


@pytest.mark.parametrize("V", [2049, 5000, 8191, 8192, 8193, 12288, 12289])
def test_equal_logits_around_one_workgroups_row(V):
    """as in the largest call; a second, lower level of equal logits lies beyond the first"""
    M, rng = 40, np.random.default_rng(V)
    u = rng.integers(0, 1 << 24, M).astype(np.float64) / (1 << 24)
    first = rng.permutation(V)[:V // 2]
    x = np.full((M, V), -1.0, dtype=np.float32)
    x[:, first] = 1.0
    order = np.concatenate([np.sort(first), np.setdiff1d(np.arange(V), first)])   # falling logits, then by index
    k = rng.integers(2, V // 2, M)
    token, prob = run(x, top_k=k, u=u)
    for m in range(M):
        assert token[m] == order[:k[m]][int(u[m] * k[m])]
    np.testing.assert_array_equal(prob, (1.0 / k).astype(np.float32))
    k = rng.integers(V // 2 + 1, V, M)
    for m, t in enumerate(run(x, top_k=k, u=u)[0]):   # all of the first level and some of the second
        assert t in order[:k[m]]
    check(x[:4], top_k=k[:4], top_p=[0.9, 0.5, 0.99, 1.0], min_p=[0, 0, 0.01, 0], u=u[:4])


@pytest.mark.parametrize("limits", LIMITS)
@pytest.mark.parametrize("V", [8192, 8500, 12287, 12288, 12289])
def test_random_rows_around_one_workgroups_row(V, limits):
    x, rng = rows(V, 3, V)
    has = lambda n: n in limits or limits == "all"
    check(x, rng.uniform(0.4, 2.5, 3), rng.integers(1, 3000, 3) if has("k") else None, rng.uniform(0.3, 1, 3) if has("p") else None,
          rng.uniform(0, 0.05, 3) if has("min") else None, rng.random(3))


@pytest.mark.parametrize("M,V", [(1, 20000), (7, 40000), (60, 33000)])
def test_one_workspace_for_the_head_and_the_sampler(M, V):
    """lm_head_topk keeps its statistics behind the tickets that lm_head_sample, the linears and the attention count with: one initialisation serves them all"""
    K, top_k = 256, 3
    gen = torch.Generator(device=DEV).manual_seed(M)
    half = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device=DEV) * std).half()
    x, W = half(M, K), half(V, K, std=0.1)
    packed = torch.empty(B.lm_head_packed_bytes(V, K), dtype=torch.uint8, device=DEV)
    B.lm_head_pack(W, packed, V, K)
    rng = np.random.default_rng(M)
    f = lambda a, t=torch.float32: torch.as_tensor(a, dtype=t, device=DEV)
    limits = f(rng.uniform(0.5, 1.5, M)), f(rng.integers(1, 400, M), torch.int32), f(rng.uniform(0.5, 1.0, M)), f(rng.uniform(0, 0.05, M)), f(rng.random(M))

    def step(head_ws, sample_ws):
        logits, idx = torch.empty(M, V, device=DEV), torch.empty(M, top_k, dtype=torch.int32, device=DEV)
        lp, token, prob = torch.empty(M, top_k, device=DEV), torch.full((M,), -1, dtype=torch.int32, device=DEV), torch.full((M,), -1.0, device=DEV)
        B.lm_head_topk(x, packed, M, V, K, top_k, logits, idx, lp, head_ws)
        B.lm_head_sample(logits, M, V, *limits, token, prob, sample_ws)
        torch.cuda.synchronize()
        return logits, idx, lp, token, prob

    head_bytes, sample_bytes = B.lm_head_workspace_bytes(M, V, K, top_k), B.lm_head_sample_workspace_bytes(M, V)
    want = step(torch.empty(head_bytes, dtype=torch.uint8, device=DEV), B.new_workspace(sample_bytes))
    assert (want[3] >= 0).all()
    shared = B.new_workspace(max(head_bytes, sample_bytes))
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(step(shared, shared), want))
        assert not shared[:16384].any()
    exact = B.new_workspace(head_bytes)
    B.lm_head_topk(x, packed, M, V, K, top_k, *(torch.empty_like(t) for t in want[:3]), exact)
    assert not exact[:16384].any()


@pytest.mark.parametrize("limits", ["p", "kp", "all"])
@pytest.mark.parametrize("V,T", [(128256, 1.0), (262144, 1.0), (262144, 1.5), (12000, 1.0)])
@pytest.mark.parametrize("p", [0.95, 0.999, 0.9999, 0.99999])
def test_top_p_next_to_one(V, T, p, limits):
    """Thousands of small weights lie around the border.  Half of the rows fall with the index, so that a uniform number next to one draws the border's
    token.  The definition leaves a border open by b = V (2^-45 + e^-31) of the row's weight, in top_p and in u: the token has to be one that a cut and a draw
    within b give."""
    print(f"sample V={V} T={T} top_p={p} {limits}", flush=True)
    M = 6
    x, rng = rows(V, M, V)
    x[M // 2:] = -np.sort(-x[M // 2:], axis=1)
    u = np.array([0.0, 0.5, 1 - 2.0 ** -24, 0.3125, 1 - 2.0 ** -20, 1 - 2.0 ** -24])
    k = np.full(M, V * 3 // 4) if limits != "p" else None
    q = 1e-7 if limits == "all" else None
    token, prob = run(x, T, k, p, q, u)
    b, p32, q32 = V * (2.0 ** -45 + 3.5e-14), float(np.float32(p)), float(np.float32(1e-7))
    for m in range(M):
        order = np.argsort(-x[m], kind="stable")[:V if k is None else k[m]]
        w = np.exp((x[m][order].astype(np.longdouble) - np.longdouble(x[m].max())) / T)
        w[w < np.exp(np.longdouble(-31))] = 0
        before = (np.cumsum(w) - w) / w.sum()
        found = []
        for cut in (p32 - b, p32 + b):
            kept = order[:max(1, int((before < cut).sum()))]
            share = w[:len(kept)].copy()
            if q is not None:
                share[1:][share[1:] < q32] = 0
            by_index = np.argsort(kept)
            kept, share = kept[by_index], share[by_index]
            upto = np.cumsum(share) / share.sum()
            last = np.flatnonzero(share)[-1]
            for draw in (u[m] - b, u[m] + b):
                found.append(int(kept[min(int(np.searchsorted(upto, draw, side="right")), last)]))
            place = int(np.searchsorted(kept, token[m]))
        assert min(found) <= token[m] <= max(found) and kept[place] == token[m] and share[place] > 0, (m, token[m], found)
        want = float(share[place] / share.sum())
        assert abs(prob[m] - want) <= want * (2.0 ** -23 + 4 * b), (m, prob[m], want)
