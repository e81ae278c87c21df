"""GPU: causal attention of packed sequences against the fp64 oracle, at the lengths, masks and contents where it can go wrong."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
SENTINEL = 7.0


class Batch:
    """sequences (queries, keys), packed queries with `pad` rows behind them, keys in a cache with `gap` rows between (gap None: they lie as the queries do)"""

    def __init__(self, seed, lens, Hq, Hkv, D, gap=3, pad=2, q_std=1.2):
        rng = np.random.default_rng(seed)
        self.lens, self.Hq, self.Hkv, self.D, self.scale = lens, Hq, Hkv, D, D ** -0.5
        self.rows = sum(n for n, _ in lens) + pad
        self.q_start = np.cumsum([0] + [n for n, _ in lens]).astype(np.int32)
        self.k_start = self.k_len = None
        k_rows = self.rows
        if gap is not None:
            ends = np.cumsum([gap] + [t + gap for _, t in lens])
            self.k_start, self.k_len, k_rows = ends[:-1].astype(np.int32), np.array([t for _, t in lens], dtype=np.int32), int(ends[-1])
        self.q = (rng.standard_normal((self.rows, Hq, D)) * q_std).astype(np.float16)
        self.k, self.v = (rng.standard_normal((k_rows, Hkv, D)).astype(np.float16) for _ in range(2))

    def run(self, max_q=None, max_k=None, ws=None, out=None):
        q, k, v, starts = dev(self.q), dev(self.k), dev(self.v), dev(self.q_start)
        ks, kl = (None, None) if self.k_len is None else (dev(self.k_start), dev(self.k_len))
        most = max_q or max(max(n for n, _ in self.lens), 1), max_k or max(max(t for _, t in self.lens), 1)
        size = B.w4a16_prompt_attn_workspace_bytes(self.rows, len(self.lens), *most, self.Hq, self.Hkv, self.D)
        ws = B.new_workspace(size) if ws is None else ws
        ws[16384:].fill_(0xFF)   # NaN in whatever is read before it is written
        out = torch.full_like(q, SENTINEL) if out is None else out
        print(f"prompt_attn {self.lens[:6]} x{len(self.lens)} heads {self.Hq}/{self.Hkv} D {self.D} most {most}", flush=True)
        B.w4a16_prompt_attn(q, k, v, starts, ks, kl, out, len(self.lens), self.rows, k.shape[0], *most, self.Hq, self.Hkv, self.D, self.scale, ws)
        torch.cuda.synchronize()
        return out.cpu().numpy()

    def check(self, got=None, **kw):
        got = self.run(**kw) if got is None else got
        ref, spread = R.prompt_attn(self.q, self.k, self.v, self.q_start, self.k_start, self.k_len, self.scale, np.full(self.q.shape, SENTINEL))
        close(got, ref, spread, max(t for _, t in self.lens), self.scale * self.D * np.abs(self.q.astype(np.float64)).max() * 6)
        return got


def close(got, ref, spread, keys, most):
    """the output's rounding, half a step (2^-11 of it, 2^-25 below the normal range); the probabilities' roundings, 2^-11 of each and 2^-25 of the
    largest for those below the normal range, which may be 2^-8 of it; fp32: products and their exponent, whose error is below 2^-22 of the largest
    score (`most` bounds |score|), sums and the final quotient below 2^-20"""
    fine = np.isfinite(ref)
    assert (np.isfinite(got) == fine).all()
    err = np.abs(got.astype(np.float64) - ref)[fine]
    bound = 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + (2.0 ** -11 + 2.0 ** -20 + 2.0 ** -22 * most) * spread + keys * 2.0 ** -17 * 2.0 ** -8
    assert (err <= bound[fine]).all(), (err / bound[fine]).max()


HEADS = [(8, 2), (4, 4), (7, 1), (12, 3), (16, 16), (10, 5)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n, T", [(1, 1), (1, 2), (2, 2), (1, 63), (1, 64), (1, 65), (3, 64), (31, 31), (33, 33), (64, 64), (65, 130), (100, 257), (129, 129), (200, 1000), (5, 4000)])
def test_one_sequence(n, T, D):
    Batch(n * 7 + T, [(n, T)], *HEADS[(n + T) % len(HEADS)], D).check()


@pytest.mark.parametrize("Hq, Hkv", HEADS + [(28, 4), (64, 8), (64, 1)])
def test_packed_sequences_of_different_lengths(Hq, Hkv):
    lens = [(1, 1), (70, 70), (1, 300), (3, 2), (33, 95), (17, 17), (1, 64), (130, 131), (0, 40), (2, 0), (40, 7)]
    Batch(Hq * 100 + Hkv, lens, Hq, Hkv, 128 if Hq % 8 else 64).check()


@pytest.mark.parametrize("B_", [65, 130])
def test_many_sequences(B_):
    rng = np.random.default_rng(B_)
    Batch(B_, [(int(n), int(n + p)) for n, p in zip(rng.integers(1, 9, B_), rng.integers(0, 40, B_))], 8, 2, 64).check()


@pytest.mark.parametrize("lens", [[(1, 500), (1, 1), (1, 0), (1, 77)], [(2, 900), (4, 33), (1, 129)], [(1, 3000)]])
@pytest.mark.parametrize("Hq, Hkv, D", [(8, 8, 128), (32, 8, 128), (14, 2, 64), (64, 2, 128)])
def test_single_tokens_of_a_batch(lens, Hq, Hkv, D):
    Batch(len(lens) + Hq, lens, Hq, Hkv, D).check()


@pytest.mark.parametrize("lens", [[(1, 1)], [(5, 5), (40, 40), (1, 1), (0, 0), (100, 100)]])
def test_keys_that_lie_as_the_queries_do(lens):
    Batch(9, lens, 8, 2, 128, gap=None).check()


def test_what_a_row_does_not_see_may_be_anything():
    """rows between the sequences, and inside one everything behind a row: NaN and infinities there reach nobody who does not see them"""
    for n, T, D in ((40, 40, 128), (3, 200, 128), (70, 70, 64), (1, 90, 128)):
        b = Batch(5 + n, [(n, T), (n, T)], 8, 2, D)
        clean = Batch(5 + n, [(n, T), (n, T)], 8, 2, D).run()
        outside = np.ones(b.k.shape[0], dtype=bool)
        for s, t in zip(b.k_start, b.k_len):
            outside[s:s + t] = False
        b.k[outside], b.v[outside] = np.nan, np.inf
        np.testing.assert_array_equal(b.run(), clean)
        # the last key of the second sequence: seen by its last query alone
        at = b.k_start[1] + T - 1
        b.v[at, 0, 3], b.v[at, 1, 5], b.v[at, 1, D - 1] = np.nan, np.inf, -np.inf
        got, ref = b.run(), clean.copy()
        last = 2 * n - 1
        assert np.isnan(got[last, :4, 3]).all() and (got[last, 4:, 5] == np.inf).all() and (got[last, 4:, D - 1] == -np.inf).all()
        ref[last, :4, 3], ref[last, 4:, 5], ref[last, 4:, D - 1] = got[last, :4, 3], got[last, 4:, 5], got[last, 4:, D - 1]
        np.testing.assert_array_equal(got, ref)
        b.v[at], b.k[at, 0, 0] = 0, np.nan      # a key that is no number: the one row that sees it, nobody else
        got = b.run()
        assert np.isnan(got[last, :4]).all() and np.isfinite(got[last, 4:]).all() and np.isfinite(got[:last]).all()
        np.testing.assert_array_equal(got[:last], clean[:last])


def test_rows_whose_scores_are_infinite():
    b = Batch(11, [(3, 70)], 4, 4, 128)
    b.q = np.abs(b.q)
    b.k[b.k_start[0]:b.k_start[0] + 70, 1, 0] = -np.inf          # every score of head 1
    b.k[b.k_start[0] + 68, 2, 0] = -np.inf                      # one key of head 2: no weight
    b.k[b.k_start[0] + 69, 3, 0] = np.inf                       # seen by the last row: no number
    got = b.run()
    assert np.isnan(got[:3, 1]).all() and np.isnan(got[2, 3]).all() and np.isfinite(got[:2, 3]).all()
    b.check(got)


def test_scores_of_any_size():
    for std in (1e-4, 30.0, 3000.0):
        b = Batch(12, [(50, 300)], 8, 2, 128, q_std=std)
        if std > 100:   # the largest score takes everything: a probability is 0 or 1 where the scores are apart
            got = b.run()
            ref, _ = R.prompt_attn(b.q, b.k, b.v, b.q_start, b.k_start, b.k_len, b.scale, np.full(b.q.shape, SENTINEL))
            # an error of 2^-22 of scores up to 3000 sqrt(128) 5 is up to 0.04 in the exponent
            assert np.abs(got - ref).max() <= 0.05 * np.abs(b.v.astype(np.float64)).max()
        else:
            b.check()


def test_sequences_that_do_not_lie_in_the_buffers_are_left_out():
    good = Batch(13, [(5, 9), (6, 20), (7, 7)], 8, 2, 128)
    want = good.run()
    for field, at, value in (("k_start", 1, -1), ("k_start", 1, 2 ** 31 - 1), ("k_len", 1, 1000), ("k_len", 1, -5), ("k_start", 1, 40)):
        b = Batch(13, [(5, 9), (6, 20), (7, 7)], 8, 2, 128)
        getattr(b, field)[at] = value
        got = b.run()
        assert (got[5:11] == SENTINEL).all()
        np.testing.assert_array_equal(got[:5], want[:5])
        np.testing.assert_array_equal(got[11:], want[11:])
    b = Batch(13, [(5, 9), (6, 20), (7, 7)], 8, 2, 128)
    b.q_start[3] = 10000
    np.testing.assert_array_equal(b.run()[:11], want[:11])
    b.q_start[:] = [0, 20, 11, 18]      # 20 -> 11 runs backwards: left out; 0 .. 19 with 9 keys; 11 .. 17 are named twice, by no more than this
    b.run()
    b.q_start[:] = [-3, 5, 11, 18]
    got = b.run()
    assert (got[:5] == SENTINEL).all()
    np.testing.assert_array_equal(got[5:18], want[5:18])


@pytest.mark.parametrize("lens, Hq, Hkv", [([(1, 2000), (1, 30)], 8, 8), ([(100, 2500)], 8, 2), ([(300, 300)], 16, 2)])
def test_the_stated_maxima_change_roundings_only(lens, Hq, Hkv):
    for max_q, max_k in ((None, None), (1, 1), (4096, 65536)):
        Batch(14, lens, Hq, Hkv, 128).check(max_q=max_q, max_k=max_k)


def test_a_long_prompt_against_its_pieces():
    """rows of a long prompt, and the same rows asked for alone"""
    n, Hq, Hkv, D = 5000, 8, 2, 128
    b = Batch(15, [(n, n)], Hq, Hkv, D)
    got = b.run()
    for i in (0, 1, 63, 64, 65, 1023, 2500, 4095, 4999):
        one = Batch(15, [(n, n)], Hq, Hkv, D)
        one.lens, one.rows, one.q = [(1, i + 1)], 1, b.q[i:i + 1]
        one.q_start, one.k_len = np.array([0, 1], dtype=np.int32), np.array([i + 1], dtype=np.int32)
        out = one.check()
        ref, spread = R.prompt_attn(one.q, one.k, one.v, one.q_start, one.k_start, one.k_len, one.scale, out)
        close(got[i:i + 1], ref, spread, n, one.scale * D * np.abs(one.q.astype(np.float64)).max() * 6)


def test_a_cache_beyond_4_gib():
    rows, Hkv, D, n, T = 2 ** 32 // (8 * 128 * 2) + 500, 8, 128, 3, 150
    b = Batch(16, [(n, T)], 16, Hkv, D)
    want = b.run()
    k = torch.empty(rows, Hkv, D, dtype=torch.float16, device=DEV)
    v = torch.empty(rows, Hkv, D, dtype=torch.float16, device=DEV)
    at = rows - T - 4
    s = b.k_start[0]
    k[at:at + T], v[at:at + T] = dev(b.k[s:s + T]), dev(b.v[s:s + T])
    out = torch.full((b.rows, 16, D), SENTINEL, dtype=torch.float16, device=DEV)
    ws = B.new_workspace(B.w4a16_prompt_attn_workspace_bytes(b.rows, 1, n, T, 16, Hkv, D))
    print("a cache of 4.3 GB", flush=True)
    B.w4a16_prompt_attn(dev(b.q), k, v, dev(b.q_start), dev(np.array([at], dtype=np.int32)), dev(b.k_len), out, 1, b.rows, rows, n, T, 16, Hkv, D, b.scale, ws)
    np.testing.assert_array_equal(out.cpu().numpy(), want)


@pytest.mark.parametrize("lens, Hq", [([(1, 700), (1, 90)], 8), ([(60, 900), (3, 3)], 16), ([(700, 700)], 8)])
def test_graph_replays_and_another_stream(lens, Hq):
    b = Batch(17, lens, Hq, 2, 128)
    want = b.run()
    args = [dev(t) for t in (b.q, b.k, b.v, b.q_start, b.k_start, b.k_len)]
    most = max(n for n, _ in lens), max(t for _, t in lens)
    ws = B.new_workspace(B.w4a16_prompt_attn_workspace_bytes(b.rows, len(lens), *most, Hq, 2, 128))
    outs = [torch.full((b.rows, Hq, 128), SENTINEL, dtype=torch.float16, device=DEV) for _ in range(2)]
    call = lambda out: B.w4a16_prompt_attn(*args, out, len(lens), b.rows, b.k.shape[0], *most, Hq, 2, 128, b.scale, ws)
    call(outs[0])
    torch.cuda.synchronize()
    graphs = []
    for out in outs:      # two graphs on one workspace, replayed in turn on one stream
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(out)
        graphs.append(g)
    for turn in range(4):
        for out in outs:
            out.fill_(SENTINEL)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            np.testing.assert_array_equal(out.cpu().numpy(), want)
        call(outs[0])     # eager work between the replays
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs[1].fill_(SENTINEL)
        call(outs[1])
    side.synchronize()
    np.testing.assert_array_equal(outs[1].cpu().numpy(), want)
    # other lengths in the same buffers reach the captured call: it reads them on the device
    args[5][0] -= 1
    graphs[0].replay()
    b.k_len[0] -= 1
    np.testing.assert_array_equal(outs[0].cpu().numpy(), b.run())


def test_many_calls_give_the_same_bits():
    b = Batch(18, [(1, 3000), (30, 1500), (1, 10)], 16, 4, 128)
    want = b.run()
    for _ in range(10):
        np.testing.assert_array_equal(b.run(), want)


@pytest.mark.parametrize("lens, Hq, Hkv, D", [([(1, 700), (1, 33), (2, 300)], 8, 2, 128), ([(1, 900)] * 5, 8, 8, 64), ([(200, 200), (100, 350)], 8, 2, 128), ([(130, 130), (70, 71)], 8, 2, 64),
                                              ([(600, 4000)], 16, 2, 128), ([(2100, 2100)], 32, 8, 128)])
def test_keys_that_arrive_late(lens, Hq, Hkv, D):
    """caches emptied before every call: a step that does not wait for its keys and values uses what was there before"""
    rows, keys = sum(n for n, _ in lens), sum(T for _, T in lens)
    g = torch.Generator(device=DEV).manual_seed(keys)
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV).half()
    q, k, v = rand(rows, Hq, D), rand(keys, Hkv, D), rand(keys, Hkv, D)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    q_start, k_start = np.cumsum([0] + [n for n, _ in lens]), np.cumsum([0] + [T for _, T in lens])
    most = max(n for n, _ in lens), max(T for _, T in lens)
    ws = B.new_workspace(B.w4a16_prompt_attn_workspace_bytes(rows, len(lens), *most, Hq, Hkv, D))
    where = ints(q_start.tolist()), ints(k_start[:-1].tolist()), ints([T for _, T in lens])
    other = torch.zeros(1 << 28, dtype=torch.int32, device=DEV)   # 1 GiB
    first = None
    for call in range(12):
        out = torch.full((rows, Hq, D), 9.0, dtype=torch.float16, device=DEV)
        if call:
            other.add_(1)
        B.w4a16_prompt_attn(q, k, v, *where, out, len(lens), rows, keys, *most, Hq, Hkv, D, D ** -0.5, ws)
        if first is None:
            first = out
        assert torch.equal(out, first), call


@pytest.mark.parametrize("lens, Hq, Hkv, D", [([(40, 40), (70, 70)], 8, 2, 128), ([(150, 150), (90, 200)], 14, 2, 64), ([(100, 2500), (60, 1000)], 8, 2, 128), ([(100, 2500), (60, 1000)], 14, 2, 64),
                                              ([(3, 600), (2, 333)], 8, 2, 128), ([(2100, 2100)], 64, 8, 128)])
def test_one_value_that_is_not_finite(lens, Hq, Hkv, D):
    """in kernels for few rows, tiles of 128 and 256 rows, whole and cut: it reaches the rows that see it, in its place, and nothing else"""
    b = Batch(21, lens, Hq, Hkv, D)
    clean = b.run()
    n, T = lens[-1]
    key, group = T - (n + 1) // 2, Hq // Hkv   # seen by the later half of the last sequence's queries
    b.v[b.k_start[-1] + key, 0, 3], b.v[b.k_start[-1] + key, Hkv - 1, D - 1] = np.inf, np.nan
    got, want = b.run(), clean.copy()
    sees = slice(b.q_start[-2] + key - (T - n), b.q_start[-1])
    assert not np.isfinite(got[sees, :group, 3]).any() and not np.isfinite(got[sees, -group:, D - 1]).any()
    want[sees, :group, 3], want[sees, -group:, D - 1] = got[sees, :group, 3], got[sees, -group:, D - 1]
    np.testing.assert_array_equal(got, want)


def test_rows_of_the_largest_tiles():
    """prompts long and many enough for tiles of 256 rows, which begin and end inside queries of odd groups: rows of them, and the same rows asked for alone"""
    for lens, Hq, Hkv in (([(2100, 2100)], 64, 8), ([(3500, 3700)], 40, 8)):
        n, T = lens[0]
        b = Batch(22, lens, Hq, Hkv, 128)
        got = b.run()
        assert (got[n:] == SENTINEL).all()
        for i in (0, 1, 31, 32, 51, 52, 700, n - 33, n - 1):
            one = Batch(22, lens, Hq, Hkv, 128)
            one.lens, one.rows, one.q = [(1, T - n + i + 1)], 1, b.q[i:i + 1]
            one.q_start, one.k_len = np.array([0, 1], dtype=np.int32), np.array([T - n + i + 1], dtype=np.int32)
            ref, spread = R.prompt_attn(one.q, one.k, one.v, one.q_start, one.k_start, one.k_len, one.scale, np.zeros(one.q.shape))
            close(got[i:i + 1], ref, spread, T, one.scale * 128 * np.abs(one.q.astype(np.float64)).max() * 6)


@pytest.mark.parametrize("where", [0, 40, 69])
def test_a_cut_tile_among_many_sequences(where):
    """more sequences than a wavefront reads at a time, one of them long enough to be cut, empty ones between"""
    lens = [(i % 3, 1 + 7 * i % 150) for i in range(70)]
    lens[where] = (100, 9000)
    Batch(23 + where, lens, 8, 2, 128).check()
