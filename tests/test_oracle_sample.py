"""The sampling oracle against small cases worked by hand and by brute force."""
import itertools

import numpy as np
import pytest

from oracle import sample


def test_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.3, 0.2]))
    assert sample(x, 0.05)[0] == 0 and sample(x, 0.49)[0] == 1 and sample(x, 0.51)[0] == 2 and sample(x, 0.99)[0] == 3
    token, probs, ids, _ = sample(x, 0.6, top_k=2)
    assert token == 2 and ids.tolist() == [1, 2] and np.allclose(probs, [0, 4 / 7, 3 / 7, 0])
    assert sample(x, 0.5, top_p=0.65)[2].tolist() == [1, 2]
    assert sample(x, 0.5, top_p=0.75)[2].tolist() == [1, 2, 3]
    assert sample(x, 0.5, top_k=3, top_p=0.75)[2].tolist() == [1, 2]        # of 0.9: 0.7 is past 0.675
    assert sample(x, 0.5, min_p=0.6)[2].tolist() == [1, 2]
    assert sample(x, 0.5, temperature=0.0)[0] == 1 and sample(x, 0.5, top_p=0.0)[0] == 1
    assert np.allclose(sample(x, 0.5, temperature=0.5)[1], np.array([1, 16, 9, 4]) / 30)


def test_equal_logits_go_to_the_lower_ids():
    assert sample(np.zeros(6), 0.5, top_k=2)[2].tolist() == [0, 1]
    assert sample(np.zeros(4), 0.5, top_p=0.5)[2].tolist() == [0, 1]
    assert sample(np.zeros(4), 0.5, top_p=0.51)[2].tolist() == [0, 1, 2]
    assert sample([0, 1, 1, 0, 1.0], 0.0, temperature=0)[0] == 1


def test_masked_rows():
    assert sample([-np.inf] * 3, 0.3)[0] == -1
    assert sample([np.nan, -np.inf, 1.0], 0.3)[0] == 2
    assert sample([np.inf, 0.0, np.inf], 0.6)[0] == 2


@pytest.mark.parametrize("seed", range(6))
def test_by_brute_force(seed):
    """The shortest run from the front that each filter allows, by trying all."""
    rng = np.random.default_rng(seed)
    x = rng.integers(-3, 4, 7) * 0.5
    for T, k, p, m in itertools.product((0.7, 1.0), (0, 1, 3), (0.4, 0.8, 1.0), (0.0, 0.3)):
        order = sorted(range(7), key=lambda i: (-x[i], i))
        w = [np.exp((x[i] - max(x)) / T) for i in order]
        left = k if k > 0 else 7
        n_p = next(n for n in range(1, left + 1) if p >= 1 and n == left or p < 1 and sum(w[:n]) >= p * sum(w[:left]))
        n_m = max([n for n in range(1, 8) if all(y >= m for y in w[:n])])
        stay = sorted(order[:min(left, n_p, n_m)])
        token, probs, ids, _ = sample(x, 0.37, T, k, p, m)
        assert ids.tolist() == stay and abs(probs.sum() - 1) < 1e-12
        assert np.cumsum(probs)[token] > 0.37 - 1e-12 and (token == stay[0] or np.cumsum(probs)[token - 1] <= 0.37 + 1e-12)
