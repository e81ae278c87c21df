"""GPU: each kernel that the planners of w4a16_prompt_attn and w8a8_gemm pick, against the oracle and in the calls that can go wrong: values that are not
finite, keys that arrive late, sequences that are left out, rows without keys, graphs and other streams.  tests/test_prompt_plans_host.py holds that the
cases take the kernels that they are named for."""
import numpy as np
import pytest
import torch

from paper_2505_22179_amd import binding as B
from tests.test_gpu_prompt_attn import Batch, SENTINEL, dev
from tests.test_gpu_w8a8 import Linear

pytestmark = pytest.mark.gpu
DEV = "cuda"
# sequences (queries, keys), query heads, KV heads, D
PATHS = {
    "few, D 128": ([(1, 700), (2, 33), (1, 1500)], 8, 2, 128),
    "few, D 64": ([(1, 700), (2, 33), (1, 1500)], 14, 2, 64),
    "whole 128, D 128": ([(100, 100), (40, 90), (150, 200)], 8, 2, 128),
    "whole 128, D 64": ([(100, 100), (40, 90), (150, 200)], 14, 2, 64),
    "whole 256, D 128": ([(2100, 2100), (2050, 2060), (2200, 2200)], 64, 8, 128),
    "cut, D 128": ([(100, 9000), (40, 3000), (60, 5000)], 8, 2, 128),
    "cut, D 64": ([(100, 9000), (40, 3000), (60, 5000)], 14, 2, 64),
}
SMALL = [p for p in PATHS if p != "whole 256, D 128"]   # the others' outputs are compared with the oracle whole, those of this one with its own
# (streamed or tiles, tokens, channels, walk shared): M, N, K
PRODUCTS = {
    (0, 16, 16, False): [(3, 264, 1040), (16, 1000, 336)],
    (0, 32, 16, False): [(17, 520, 2064), (31, 1032, 80)],
    (0, 32, 32, False): [(25, 6152, 1040), (32, 6168, 208)],
    (0, 64, 16, False): [(48, 4104, 512), (63, 264, 1296)],
    (0, 64, 32, False): [(60, 6152, 528), (33, 6184, 272)],
    (1, 64, 128, False): [(72, 168, 80), (127, 1032, 400)],
    (1, 64, 128, True): [(89, 136, 1040), (60, 1032, 12304)],
    (1, 128, 128, False): [(172, 168, 96), (300, 4104, 1024)],
    (1, 128, 128, True): [(130, 264, 4112), (700, 1000, 4624)],
    (1, 128, 256, False): [(391, 8200, 64), (421, 8424, 208), (397, 8712, 400)],
    (1, 256, 256, False): [(1028, 7416, 64), (1560, 4872, 208), (921, 8264, 400)],
}


def plan_of(lens, Hq, Hkv, D, pad=2):
    return B.w4a16_prompt_attn_plan_describe(sum(n for n, _ in lens) + pad, len(lens), max(n for n, _ in lens), max(t for _, t in lens), Hq, Hkv, D)


@pytest.mark.parametrize("lens, Hq, Hkv, D", [([(100, 9000)], 14, 2, 64), ([(100, 9000)], 8, 2, 64), ([(100, 9000), (60, 4000)], 8, 2, 64), ([(33, 12001)], 28, 4, 64), ([(200, 7777)], 3, 3, 64),
                                              ([(1, 9000), (100, 4000), (1, 1)], 14, 2, 64)] + [PATHS[p] for p in SMALL])
def test_against_the_oracle(lens, Hq, Hkv, D):
    Batch(51 + len(lens), lens, Hq, Hkv, D).check()


@pytest.mark.parametrize("D, Hq", [(64, 14), (64, 8), (128, 8)])
@pytest.mark.parametrize("where", [0, 40, 69])
def test_a_cut_tile_among_many_sequences(where, D, Hq):
    lens = [(i % 3, 1 + 7 * i % 150) for i in range(70)]
    lens[where] = (100, 9000)
    assert plan_of(lens, Hq, 2, D)[0] == 2
    Batch(52 + where, lens, Hq, 2, D).check()


@pytest.mark.parametrize("path", PATHS)
def test_one_value_that_is_not_finite(path):
    """it reaches the rows that see it, in its place, and nothing else"""
    lens, Hq, Hkv, D = PATHS[path]
    b = Batch(53, lens, Hq, Hkv, D)
    clean = b.run()
    n, T = lens[-1]
    key, group = T - (n + 1) // 2, Hq // Hkv   # seen by the later half of the last sequence's queries
    b.v[b.k_start[-1] + key, 0, 3], b.v[b.k_start[-1] + key, Hkv - 1, D - 1] = np.inf, np.nan
    got, want = b.run(), clean.copy()
    sees = slice(b.q_start[-2] + key - (T - n), b.q_start[-1])
    assert not np.isfinite(got[sees, :group, 3]).any() and not np.isfinite(got[sees, -group:, D - 1]).any()
    want[sees, :group, 3], want[sees, -group:, D - 1] = got[sees, :group, 3], got[sees, -group:, D - 1]
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("path", PATHS)
def test_keys_that_arrive_late(path):
    """caches emptied before every call: a step that does not wait for its keys and values uses what was there before"""
    lens, Hq, Hkv, D = PATHS[path]
    b = Batch(54, lens, Hq, Hkv, D)
    first, other = b.run(), torch.zeros(1 << 28, dtype=torch.int32, device=DEV)   # 1 GiB
    args = [dev(t) for t in (b.q, b.k, b.v, b.q_start, b.k_start, b.k_len)]
    most = max(n for n, _ in lens), max(t for _, t in lens)
    ws = B.new_workspace(B.w4a16_prompt_attn_workspace_bytes(b.rows, len(lens), *most, Hq, Hkv, D))
    for call in range(8):
        out = torch.full((b.rows, Hq, D), SENTINEL, dtype=torch.float16, device=DEV)
        other.add_(1)
        B.w4a16_prompt_attn(*args, out, len(lens), b.rows, b.k.shape[0], *most, Hq, Hkv, D, b.scale, ws)
        np.testing.assert_array_equal(out.cpu().numpy(), first)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("field, at, value", [("k_start", 1, -1), ("k_start", 1, 2 ** 31 - 1), ("k_len", 1, 10 ** 6), ("k_len", 1, -5), ("k_len", 0, 2 ** 31 - 1), ("q_start", 3, 10 ** 6),
                                              ("q_start", 2, 2 ** 31 - 1), ("q_start", 2, -4), ("q_start", 0, -3), ("q_start", 0, -2 ** 31)])
def test_sequences_that_do_not_lie_in_the_buffers_are_left_out(path, field, at, value):
    """their rows keep what they held, and the others are the oracle's (where it is slow: their own of a call in which the batch is as it should be)"""
    lens, Hq, Hkv, D = PATHS[path]
    b = Batch(55, lens, Hq, Hkv, D)
    want = b.run() if path not in SMALL else None
    rows = b.q_start.copy()
    getattr(b, field)[at] = value
    if want is None:
        b.check()
        return
    got = b.run()
    out_of_it = {("k_start", 1): [1], ("k_len", 1): [1], ("k_len", 0): [0], ("q_start", 3): [2], ("q_start", 2): [1, 2], ("q_start", 0): [0]}[field, at]
    for s in out_of_it:
        assert (got[rows[s]:rows[s + 1]] == SENTINEL).all()
        want[rows[s]:rows[s + 1]] = SENTINEL
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("Hq, D", [(8, 128), (14, 64)])
@pytest.mark.parametrize("lens", [[(600, 40), (100, 9000)], [(100, 9000), (600, 40)], [(300, 0), (100, 9000), (900, 1)]])
def test_tiles_of_which_no_row_sees_a_key(lens, Hq, D):
    """more queries than keys beside a long sequence, in tiles that are cut and joined; and alone, in whole tiles"""
    assert plan_of(lens, Hq, 2, D)[0] == 2
    Batch(56, lens, Hq, 2, D).check()
    alone = [s for s in lens if s[1] < 100]
    assert plan_of(alone, Hq, 2, D)[0] == 1
    Batch(57, alone, Hq, 2, D).check()


@pytest.mark.parametrize("path", PATHS)
def test_sequences_whose_rows_run_backwards(path):
    """0 .. n, back, and on from there: the one that runs backwards is left out, rows in no sequence keep what they held"""
    lens, Hq, Hkv, D = PATHS[path]
    b = Batch(58, lens, Hq, Hkv, D)
    want = b.run()
    last = b.q_start[2]
    b.q_start[:] = [last, b.q_start[3], 0, b.q_start[1]]   # the third's rows with the first's keys, none, the first's rows with the third's keys
    got = b.run()
    assert (got[b.q_start[3]:last] == SENTINEL).all() and (got[b.q_start[1]:] == SENTINEL).all()
    assert np.isfinite(got).all() and (got[:b.q_start[3]] != want[:b.q_start[3]]).any()


@pytest.mark.parametrize("path", PATHS)
def test_graph_replays_and_another_stream(path):
    lens, Hq, Hkv, D = PATHS[path]
    b = Batch(59, lens, Hq, Hkv, D)
    want = b.run()
    args = [dev(t) for t in (b.q, b.k, b.v, b.q_start, b.k_start, b.k_len)]
    most = max(n for n, _ in lens), max(t for _, t in lens)
    ws = B.new_workspace(B.w4a16_prompt_attn_workspace_bytes(b.rows, len(lens), *most, Hq, Hkv, D))
    outs = [torch.full((b.rows, Hq, D), SENTINEL, dtype=torch.float16, device=DEV) for _ in range(2)]
    call = lambda out: B.w4a16_prompt_attn(*args, out, len(lens), b.rows, b.k.shape[0], *most, Hq, Hkv, D, b.scale, ws)
    call(outs[0])
    torch.cuda.synchronize()
    graphs = []
    for out in outs:      # two graphs on one workspace, replayed in turn on one stream
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(out)
        graphs.append(g)
    for _ in range(4):
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
    args[5][0] -= 1       # another length in the same buffers reaches the captured call: it reads them on the device
    graphs[0].replay()
    b.k_len[0] -= 1
    np.testing.assert_array_equal(outs[0].cpu().numpy(), b.run())


@pytest.mark.parametrize("M, N, K", [sizes for many in PRODUCTS.values() for sizes in many])
def test_products_of_every_kernel(M, N, K):
    Linear(M + N + K, M, N, K, [B.W8A8_PLAIN, B.W8A8_RMS_NORM, B.W8A8_SILU_MUL][N % 3], M % 2 == 0).check()
