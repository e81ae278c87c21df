"""GPU: rotary tables and the rotation of packed tokens against the fp64 oracle, and bit for bit against rope_append where both apply."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import binding as B
from paper_2505_22179_amd import inputs as I

pytestmark = pytest.mark.gpu
DEV = "cuda"
dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
SCALINGS = {"plain": (B.ROPE_PLAIN, 1.0, 0.0, 0.0, 0.0), "linear": (B.ROPE_LINEAR, 4.0, 0.0, 0.0, 0.0), "turns": (B.ROPE_BY_TURNS, 8.0, 1.0, 4.0, 8192.0),
            "index": (B.ROPE_BY_INDEX, 16.0, 1.0, 32.0, 4096.0), "index that meets": (B.ROPE_BY_INDEX, 2.0, 1.0, 1.0001, 7.0)}


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("first, n, R_", [(0, 1, 2), (0, 1, 128), (5, 33, 6), (0, 257, 64), (1000, 100, 130), (2 ** 20 - 40, 40, 128), (2 ** 28 - 9, 9, 32), (0, 31, 1024)])
def test_tables(first, n, R_, scaling):
    kind, factor, low, high, original = SCALINGS[scaling]
    amplitude = 1.0 if first else 1.2079
    cos, sin = (torch.full((n + 1, R_ // 2), 9.0, device=DEV) for _ in range(2))
    print(f"rope_table {first} {n} {R_} {scaling}", flush=True)
    B.rope_table(cos, sin, first, n, R_, 500000.0, kind, factor, low, high, original, amplitude)
    torch.cuda.synchronize()
    for got, ref in zip((cos, sin), R.rope_table(first, n, R_, 500000.0, kind, factor, low, high, original, amplitude)):
        got = got.cpu().numpy()
        assert (got[n:] == 9.0).all()
        # fp32 half step; the angle's roundings (frequency: exponential and blend, a few of 2^-53; product), here and in the oracle; series 2^-36
        tol = 2.0 ** -24 * np.abs(ref) + abs(amplitude) * ((first + n) * 2.0 ** -48 + 2.0 ** -35)
        assert (np.abs(got[:n].astype(np.float64) - ref) <= tol).all()


class Tokens:
    def __init__(self, seed, rows, Hq, Hkv, D, R_, interleaved, n_pos=50):
        rng = np.random.default_rng(seed)
        self.shape = rows, Hq, Hkv, D
        self.R, self.interleaved, self.n_pos = R_, interleaved, n_pos
        self.qkv = (rng.standard_normal((rows, (Hq + 2 * Hkv) * D)) * 1.5).astype(np.float16)
        self.pos = rng.integers(0, n_pos, rows).astype(np.int32)
        self.cache_rows = rows + 7
        self.slot = rng.permutation(self.cache_rows)[:rows].astype(np.int32)
        self.cos, self.sin = I.make_rope_tables(n_pos, R_)

    def buffers(self):
        rows, Hq, Hkv, D = self.shape
        return (torch.full((rows + 1, Hq, D), 77.0, dtype=torch.float16, device=DEV),
                torch.full((self.cache_rows, Hkv, D), 55.0, dtype=torch.float16, device=DEV), torch.full((self.cache_rows, Hkv, D), 66.0, dtype=torch.float16, device=DEV))

    def run(self):
        rows, Hq, Hkv, D = self.shape
        q, k, v = self.buffers()
        print(f"rope_prompt {self.shape} R {self.R} interleaved {self.interleaved}", flush=True)
        B.rope_prompt(dev(self.qkv), dev(self.pos), dev(self.cos), dev(self.sin), self.n_pos, self.R, self.interleaved,
                      None if self.slot is None else dev(self.slot), self.cache_rows, q, k, v, rows, Hq, Hkv, D)
        torch.cuda.synchronize()
        return tuple(t.cpu().numpy() for t in (q, k, v))

    def check(self):
        rows = self.shape[0]
        q0, k0, v0 = (t.cpu().numpy() for t in self.buffers())
        got = self.run()
        assert (got[0][rows:] == 77).all()
        want = R.rope_prompt(self.qkv, self.pos, self.cos, self.sin, self.R, self.interleaved, self.slot, q0[:rows], k0, v0)
        np.testing.assert_array_equal(got[2], want[2].astype(np.float16))
        most = 2 * np.abs(self.qkv.astype(np.float64)).max()
        for g, w in ((got[0][:rows], want[0]), (got[1], want[1])):   # half a step, and two fp32 roundings of terms below `most`
            assert (np.abs(g.astype(np.float64) - w) <= 2.0 ** -11 * np.abs(w) + 2.0 ** -25 + 2.0 ** -23 * most).all()
        untouched = np.setdiff1d(np.arange(self.cache_rows), [s for s in (self.slot if self.slot is not None else range(rows))])
        assert (got[1][untouched] == 55).all() and (got[2][untouched] == 66).all()
        return got


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows, Hq, Hkv, D, R_", [(1, 1, 1, 8, 2), (1, 32, 8, 128, 128), (3, 5, 1, 64, 16), (17, 28, 4, 128, 64), (9, 8, 8, 80, 80), (4, 3, 3, 72, 24), (5, 2, 1, 96, 32),
                                                  (3, 4, 2, 256, 250), (2, 2, 2, 512, 512), (300, 6, 2, 128, 96), (7, 64, 8, 40, 6)])
def test_packed_tokens(rows, Hq, Hkv, D, R_, interleaved):
    Tokens(rows + D, rows, Hq, Hkv, D, R_, interleaved).check()


def test_without_a_slot_map_tokens_have_their_own_rows():
    t = Tokens(3, 20, 8, 2, 128, 128, False)
    t.slot = None
    t.check()


def test_padding_tokens_and_positions_outside_the_tables():
    for interleaved in (False, True):
        t = Tokens(4, 12, 8, 2, 64, 32, interleaved)
        t.slot[[2, 5, 7]] = [-1, t.cache_rows, 2 ** 31 - 1]
        t.pos[[1, 5, 9]] = [-1, t.n_pos, -2 ** 31]
        q, k, v = t.check()
        assert (q[[1, 5, 9]] == 77).all() and (q[[2, 7]] != 77).any()


@pytest.mark.parametrize("M, Hq, Hkv, D", [(1, 8, 2, 128), (60, 64, 8, 128), (100, 4, 4, 80)])
def test_bits_of_rope_append(M, Hq, Hkv, D):
    t = Tokens(M, M, Hq, Hkv, D, D, False)
    P = 4
    t.slot = np.arange(P, P + M, dtype=np.int32)
    got = t.run()
    q, k, v = t.buffers()
    B.rope_append(dev(t.qkv), dev(t.pos), dev(t.cos), dev(t.sin), t.n_pos, q, k, v, M, P, Hq, Hkv, D)
    for a, b in zip(got, (q, k, v)):
        np.testing.assert_array_equal(a.view(np.uint16), b.cpu().numpy().view(np.uint16))


def test_stretched_tables_reach_the_append():
    """tables that rope_table made, in rope_append and rope_prompt"""
    M, Hq, Hkv, D, n = 6, 4, 2, 128, 64
    cos, sin = (torch.empty(n, D // 2, device=DEV) for _ in range(2))
    B.rope_table(cos, sin, 0, n, D, 500000.0, B.ROPE_BY_TURNS, 8.0, 1.0, 4.0, 8192.0)
    t = Tokens(8, M, Hq, Hkv, D, D, False, n)
    t.cos, t.sin = cos.cpu().numpy(), sin.cpu().numpy()
    t.check()


def test_graph_replays():
    t = Tokens(9, 40, 8, 2, 128, 128, True)
    want = t.run()
    args = [dev(x) for x in (t.qkv, t.pos, t.cos, t.sin)]
    slot, bufs = dev(t.slot), t.buffers()
    cos, sin = torch.empty(50, 64, device=DEV), torch.empty(50, 64, device=DEV)

    def work():
        B.rope_table(cos, sin, 0, 50, 128, 500000.0)
        B.rope_prompt(*args, t.n_pos, t.R, True, slot, t.cache_rows, *bufs, *t.shape)
    work()
    torch.cuda.synchronize()
    first = cos.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(3):
        for x, fresh in zip(bufs, t.buffers()):
            x.copy_(fresh)
        cos.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cos, first)
        for x, w in zip(bufs, want):
            np.testing.assert_array_equal(x.cpu().numpy().view(np.uint16), w.view(np.uint16))


@pytest.mark.parametrize("kind, low, high, original", [(B.ROPE_LINEAR, 0.0, 0.0, 0.0), (B.ROPE_BY_TURNS, 1.0, 4.0, 8.0), (B.ROPE_BY_INDEX, 1.0, 32.0, 64.0)])
def test_tables_of_the_largest_angles(kind, low, high, original):
    first, n, R_, factor = 2 ** 28 - 20, 20, 64, 0.125
    cos, sin = (torch.zeros(n, R_ // 2, device=DEV) for _ in range(2))
    print(f"rope_table kind {kind} from {first}", flush=True)
    B.rope_table(cos, sin, first, n, R_, 10000.0, kind, factor, low, high, original, 1.0)
    torch.cuda.synchronize()
    for got, ref in zip((cos, sin), R.rope_table(first, n, R_, 10000.0, kind, factor, low, high, original, 1.0)):
        # as above, of angles that are 1 / factor times as large
        tol = 2.0 ** -24 * np.abs(ref) + 2.0 ** 31 * 2.0 ** -48 + 2.0 ** -35
        assert (np.abs(got.cpu().numpy().astype(np.float64) - ref) <= tol).all()
