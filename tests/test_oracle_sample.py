"""Pins of the sampling oracle: worked examples, library cross-checks, frequencies over a grid of uniform numbers."""
import math

import numpy as np
import pytest
import torch

from oracle import reference as R

LN = math.log


def test_worked_examples():
    logits = [LN(1), LN(4), LN(2), LN(1)]            # probabilities 1/8, 1/2, 1/4, 1/8
    tokens = lambda **kw: [R.sample(logits, u=(i + 0.5) / 16, **kw)[0] for i in range(16)]
    assert tokens() == [0] * 2 + [1] * 8 + [2] * 4 + [3] * 2
    assert tokens(temperature=0.0) == [1] * 16 and tokens(top_p=0.0) == [1] * 16 and tokens(min_p=1.5) == [1] * 16 and tokens(top_k=1) == [1] * 16
    assert tokens(top_k=3) == [R.sample(logits[:3], u=(i + 0.5) / 16)[0] for i in range(16)]     # 0 and 3 tie: the lower index stays
    assert set(tokens(top_p=0.74)) == {1, 2} and set(tokens(top_p=0.49)) == {1} and set(tokens(top_p=0.76)) == {0, 1, 2}
    assert set(tokens(min_p=0.3)) == {1, 2} and set(tokens(min_p=0.2)) == {0, 1, 2, 3}
    # top_p counts within what top_k left: 4/6 of {1, 2}
    assert set(tokens(top_k=2, top_p=0.6)) == {1} and set(tokens(top_k=2, top_p=0.7)) == {1, 2}
    assert R.sample(logits, u=0.2)[1] == pytest.approx(0.5) and R.sample(logits, top_k=2, u=0.9)[1] == pytest.approx(1 / 3)


def test_no_tokens_infinities_and_nan():
    inf, nan = math.inf, math.nan
    assert R.sample([-inf, nan, -inf])[:2] == (0x7FFFFFFF, 0.0)
    assert R.sample([nan, 1.0, -inf], u=0.99)[0] == 1
    assert [R.sample([5.0, inf, 7.0, inf], u=u)[0] for u in (0.0, 0.49, 0.51, 0.99)] == [1, 1, 3, 3]
    assert R.sample([0.0, 1.0, 2.0], temperature=inf, u=0.1)[0] == 0


@pytest.mark.parametrize("seed", range(6))
def test_against_torch(seed):
    rng = np.random.default_rng(seed)
    V, T, k, p, m = 50, rng.uniform(0.3, 2), int(rng.integers(1, 60)), rng.uniform(0.3, 1.2), rng.uniform(0, 0.3)
    x = rng.standard_normal(V) * 2
    x[rng.integers(0, V, 20)] = 0.5     # ties
    probs = torch.softmax(torch.tensor(x) / T, 0)
    s, order = torch.sort(probs, descending=True, stable=True)
    if k < V:
        s[k:] = 0
    if p < 1:
        c = torch.cumsum(s, 0)
        s[1:][~(c[:-1] < p * c[-1])] = 0
    s[1:][s[1:] < m * s[0]] = 0
    kept = torch.zeros(V, dtype=torch.float64).scatter(0, order, s)
    cdf = torch.cumsum(kept, 0) / kept.sum()
    for u in rng.random(200):
        token, prob, margin = R.sample(x, T, k, p, m, u)
        if margin > 1e-12:
            assert token == int((cdf <= u).sum()) and prob == pytest.approx(float(kept[token] / kept.sum()), rel=1e-12)
