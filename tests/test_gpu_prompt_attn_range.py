"""GPU: attention of packed sequences where scores leave the range that fp16 probabilities and fp32 exponents have room for, in every kernel."""
import numpy as np
import pytest
import torch

from paper_2505_22179_amd import binding as B
from tests.test_gpu_prompt_attn import Batch

pytestmark = pytest.mark.gpu
# few rows; tiles of 128 rows; tiles of 128 rows that are cut into ranges of keys (they have 256); whole tiles of 256 rows
KERNELS = [([(1, 4000), (1, 33)], 8, 2, 128), ([(2, 900), (1, 60)], 8, 2, 64), ([(200, 200), (40, 90)], 8, 2, 128), ([(150, 200)], 14, 2, 64), ([(100, 9000)], 8, 2, 128),
           ([(100, 9000)], 14, 2, 64), ([(2100, 2100)], 64, 8, 128)]


def rows_of(b):
    """(row, query head, first key row, keys seen) of some forty rows of the batch, the first and last of each sequence among them"""
    for (n, T), q0, k0 in zip(b.lens, b.q_start, b.k_start):
        for i in sorted({int(x) for x in np.linspace(0, n - 1, 14)}):
            for head in {0, b.Hq // 2 + 1, b.Hq - 1}:
                yield q0 + i, head, k0, T - n + i + 1


@pytest.mark.parametrize("lens, Hq, Hkv, D", KERNELS)
@pytest.mark.parametrize("std, scale", [(300.0, None), (4000.0, None), (15000.0, None), (1.2, 1e10), (1.2, 2.0 ** 60)])
def test_scores_far_from_zero(lens, Hq, Hkv, D, std, scale):
    """finite queries and keys whose largest score, of up to 2^30 and 2^66, takes everything: outputs lie among the values of the keys that may be the
    largest.  A score is off by 128 roundings of fp32 at the most, 2^-17 of its products' magnitudes; 30 below the largest, a key weighs less than 2^-43"""
    b = Batch(31, lens, Hq, Hkv, D)
    rng = np.random.default_rng(int(std))
    b.q, b.k = (np.clip(rng.standard_normal(x.shape) * std, -60000, 60000).astype(np.float16) for x in (b.q, b.k))
    b.scale = scale or b.scale
    got = b.run().astype(np.float64)
    q, k, v = (x.astype(np.float64) for x in (b.q, b.k, b.v))
    for row, head, k0, seen in rows_of(b):
        kh, vh = k[k0:k0 + seen, head // (Hq // Hkv)], v[k0:k0 + seen, head // (Hq // Hkv)]
        s, size = kh @ q[row, head], np.abs(kh) @ np.abs(q[row, head])
        may_be = vh[s >= s.max() - 2.0 ** -16 * size.max() - 30 / b.scale]
        near = 2.0 ** -10 * np.abs(may_be).max(0) + 2.0 ** -20
        assert (got[row, head] >= may_be.min(0) - near).all() and (got[row, head] <= may_be.max(0) + near).all(), (row, head)


@pytest.mark.parametrize("lens, Hq, Hkv, D", KERNELS[:6])
def test_the_smallest_scale_weighs_all_keys_alike(lens, Hq, Hkv, D):
    b = Batch(32, lens, Hq, Hkv, D)
    b.scale = 1e-38
    b.check()


@pytest.mark.parametrize("lens, Hq, Hkv, D", KERNELS)
@pytest.mark.parametrize("orders", [12, 20, 26, 30])
def test_keys_far_above_the_others(lens, Hq, Hkv, D, orders):
    """keys `orders` binary orders above all others, whose values are 0, in every range that one wavefront or workgroup walks: what the others weigh
    makes up the output.  A probability p (the row's largest 1) is rounded by 2^-11 p, or below fp16's normal range, 2^-14 where the largest is 2^7 at least,
    by 2^-25 of 2^-7; fp32 adds 2^-20 and 2^-22 of the largest score"""
    b = Batch(33, lens, Hq, Hkv, D)
    rng = np.random.default_rng(orders)
    b.scale = 1.0
    b.q = (rng.standard_normal(b.q.shape) * 0.03).astype(np.float16)
    b.q[..., 0] = 1.0
    b.k = (rng.standard_normal(b.k.shape) * 0.5).astype(np.float16)
    b.k[..., 0] = 0
    b.v = (rng.uniform(512, 1536, b.v.shape)).astype(np.float16)
    for k0, (n, T) in zip(b.k_start, b.lens):
        high = np.arange(k0, k0 + T, 32 if n < 5 else 500)
        b.k[high, :, 0], b.v[high] = orders * np.log(2), 0
    got = b.run().astype(np.float64)
    q, k, v = (x.astype(np.float64) for x in (b.q, b.k, b.v))
    for row, head, k0, seen in rows_of(b):
        kh, vh = k[k0:k0 + seen, head // (Hq // Hkv)], v[k0:k0 + seen, head // (Hq // Hkv)]
        s = kh @ q[row, head]
        p = np.exp(s - s.max())
        want = p @ vh / p.sum()
        off = np.maximum((2.0 ** -11 + 2.0 ** -20 + 2.0 ** -22 * np.abs(s).max()) * p, 2.0 ** -32)
        bound = (off @ vh + off.sum() * want) / p.sum() + 2.0 ** -11 * want + 2.0 ** -25
        err = np.abs(got[row, head] - want)
        assert (err <= bound).all(), (row, head, (err / bound).max(), want[:3], got[row, head, :3])


@pytest.mark.parametrize("lens, Hq, Hkv, D", KERNELS)
@pytest.mark.parametrize("what", ["a query far from zero", "an infinite key"])
def test_rows_far_from_zero_leave_the_others_bits_alone(lens, Hq, Hkv, D, what):
    """the rows of a wavefront share its branches, not their arithmetic"""
    b = Batch(34, lens, Hq, Hkv, D)
    b.q, b.k = (b.q * np.float16(0.03)).astype(np.float16), (b.k * np.float16(30)).astype(np.float16)
    want = b.run()
    n, T = lens[0]
    others = np.ones((b.rows, Hq), dtype=bool)
    if what == "an infinite key":   # seen by the first sequence's last row alone
        b.k[b.k_start[0] + T - 1, :, 0] = np.inf
        others[n - 1] = False
    else:                           # one head of it
        b.q[n - 1, 1] = (b.q[n - 1, 1].astype(np.float32) * 1e6).clip(-60000, 60000).astype(np.float16)
        others[n - 1, 1] = False
    got = b.run()
    np.testing.assert_array_equal(got[others].view(np.uint16), want[others].view(np.uint16))
    assert (got[~others].view(np.uint16) != want[~others].view(np.uint16)).any()
