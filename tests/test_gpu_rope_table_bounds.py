"""GPU: entries of rope_table near the first positions, where angles are small enough to show what the series and the turns from position to position add."""
import numpy as np
import pytest
import torch

from oracle import reference as R
from paper_2505_22179_amd import binding as B

pytestmark = pytest.mark.gpu
THETA = 10000.0


@pytest.mark.parametrize("R_", [2, 6, 24, 64, 128, 160, 250, 1024])   # one to 128 turns in a row
@pytest.mark.parametrize("kind, factor", [(B.ROPE_PLAIN, 1.0), (B.ROPE_LINEAR, 0.125), (B.ROPE_LINEAR, 8.0), (B.ROPE_BY_TURNS, 8.0), (B.ROPE_BY_TURNS, 0.125), (B.ROPE_BY_INDEX, 0.125)])
def test_entries_of_small_angles(R_, kind, factor):
    """Half a step of fp32.  Series and turns: 2^-44 + 2^-46 f.  The angle p f: 2^-53 of it for its own rounding, and that of f = 2^-x, here and in the oracle:
    x has three roundings of 2^-53 and moves f by ln 2 times its own, the power two; a blend's weight t moves f by |1 - 1 / factor| times its error, which is that
    of n / (high - low), below 2 (and three roundings of its own).  All of that counted as x + 4 times 2^-51 for each side, the blend's share on top of it"""
    n, low, high, original = 515, 1.0, 4.0, 2048.0
    cos, sin = (torch.full((n + 1, R_ // 2), 9.0, device="cuda") for _ in range(2))
    print(f"rope_table R {R_} kind {kind} factor {factor}", flush=True)
    B.rope_table(cos, sin, 0, n, R_, THETA, kind, factor, low, high, original)
    torch.cuda.synchronize()
    plain, f = R.rope_frequencies(R_, THETA), R.rope_frequencies(R_, THETA, kind, factor, low, high, original)
    x = -np.log2(plain)
    off = f * (x + 4) * 2.0 ** -50
    if kind == B.ROPE_BY_TURNS:
        off += plain * abs(1 - 1 / factor) * 2 * (x + 4) * 2.0 ** -50
    pos = np.arange(n)[:, None]
    for got, ref in zip((cos, sin), R.rope_table(0, n, R_, THETA, kind, factor, low, high, original)):
        got = got.cpu().numpy().astype(np.float64)
        assert (got[n:] == 9.0).all()
        tol = 2.0 ** -24 * np.abs(ref) + pos * (off + f * 2.0 ** -52) + 2.0 ** -44 + 2.0 ** -46 * f + 2.0 ** -53   # the last: the oracle's own cosine
        err = np.abs(got[:n] - ref)
        assert (err <= tol).all(), (err / tol).max()
