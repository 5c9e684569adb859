"""Pins for the oracle's filtered distributions (oracle/filter.py): hand
cases, and independent definitions by enumeration."""
import itertools
import math

import numpy as np
import pytest

from oracle import decode as od
from oracle import filter as of


def _by_enumeration(z, T, k, p, m):
    """Kept set from the definition: an order by pairwise comparison, prefixes
    tried one by one."""
    V = len(z)
    ids = sorted(range(V), key=lambda i: (-z[i], i))
    w = [math.exp((z[i] - z[ids[0]]) / T) for i in ids]
    n = k if 0 < k < V else V
    if p < 1:
        whole = math.fsum(w[:n])
        n = next(r for r in range(1, n + 1) if math.fsum(w[:r]) >= p * whole or r == n)
    return {i for r, i in enumerate(ids[:n]) if r == 0 or w[r] >= m}


@pytest.mark.parametrize("T,k,p,m", itertools.product([0.5, 1.3], [0, 2, 5], [1.0, 0.6, 0.0],
                                                      [0.0, 0.3]))
def test_kept_set_equals_enumeration(T, k, p, m):
    rng = np.random.default_rng(5)
    for _ in range(20):
        z = np.round(rng.standard_normal(9) * 2, 1)      # some ties
        w = of.kept_weights(z, T, k, p, m)
        assert set(np.flatnonzero(w)) == _by_enumeration(list(z), T, k, p, m)


def test_hand_cases():
    z = np.log(np.array([0.1, 0.4, 0.4, 0.1]))
    assert list(np.flatnonzero(of.kept_weights(z, k=1))) == [1]          # lowest index of a tie
    assert list(np.flatnonzero(of.kept_weights(z, k=2))) == [1, 2]
    assert list(np.flatnonzero(of.kept_weights(z, p=0.39))) == [1]
    assert list(np.flatnonzero(of.kept_weights(z, p=0.7))) == [1, 2]
    assert list(np.flatnonzero(of.kept_weights(z, p=0.85))) == [0, 1, 2]
    assert list(np.flatnonzero(of.kept_weights(z, m=0.5))) == [1, 2]
    np.testing.assert_allclose(of.probs(of.kept_weights(z, k=2)), [0, 0.5, 0.5, 0])
    z = np.array([-np.inf, 1.0, np.nan, -0.0, 0.0])
    assert list(np.flatnonzero(of.kept_weights(z))) == [1, 3, 4]
    assert list(np.flatnonzero(of.kept_weights(z, k=2))) == [1, 3]
    assert of.sample(np.array([-np.inf, np.nan]), 0.5) == (0, 0.0)
    assert of.sample(np.array([np.nan, -np.inf]), 0.5) == (1, 0.0)
    assert of.sample(np.array([np.nan, np.nan]), 0.5) == (0, 0.0)


def test_without_filters_equals_softmax_sampling():
    rng = np.random.default_rng(1)
    for _ in range(50):
        z, T, u = rng.standard_normal(30) * 3, rng.uniform(0.3, 2), rng.random()
        t, pr = of.sample(z, u, T)
        p = od.softmax_t(z, T)
        assert t == od.sample_index(p, u)
        assert abs(pr - p[t]) <= 1e-14
    assert of.draw(np.array([0.0, 0.0, 1.0, 0.0, 2.0]), 0.0) == 2
    assert of.draw(np.array([1.0, 1.0, 0.0]), 1.0) == 1


def test_filtered_acceptance_keeps_the_filtered_distribution():
    """The committed token's distribution over fine grids of the draft sample,
    the test and the resample equals the filtered p; a resample from p misses."""
    rng = np.random.default_rng(3)
    V, N = 6, 400
    grid = (np.arange(N) + 0.5) / N
    p = of.probs(of.kept_weights(rng.standard_normal(V), 1.0, 4, 0.9, 0.0))
    q = of.probs(of.kept_weights(rng.standard_normal(V), 1.0, 4, 0.9, 0.0))
    got = np.zeros(V)
    nxt = np.full(V, 1.0 / V)
    for d in range(V):
        if q[d] == 0:
            continue
        for u in grid:
            A, _ = of.accept(np.stack([p, nxt]), q[None], np.array([d]), np.array([u, 0.5]))
            if A == 1:
                got[d] += q[d] / N
            else:
                res = [of.accept(np.stack([p, nxt]), q[None], np.array([d]), np.array([u, v]))[1]
                       for v in (0.05, 0.35, 0.65, 0.95)]
                rest = np.maximum(p - q, 0)
                assert all(rest[t] > 0 for t in res)
                got += q[d] / N * rest / rest.sum()
    np.testing.assert_allclose(got, p, atol=2.0 / N)


def test_accept_edges():
    p = np.array([[0.5, 0.5, 0.0], [0.0, 0.0, 1.0]])
    q = np.array([[0.5, 0.5, 0.0]])
    assert of.accept(p, q, np.array([1]), np.array([0.999, 0.3])) == (1, 2)   # p == q: always
    assert of.accept(p, q, np.array([-1]), np.array([0.0, 0.7])) == (0, 1)    # no token; p - q is 0: from p
    assert of.accept(p, q, np.array([2]), np.array([0.5, 0.2])) == (0, 0)     # outside both kept sets
