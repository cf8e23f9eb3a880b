"""Pins of the sampling oracle: hand cases, brute force and frequencies (no GPU)."""
import itertools
import math

import numpy as np
import pytest

from oracle import rules as RU
from oracle import sampling as SA

L = np.log(np.array([0.1, 0.4, 0.2, 0.25, 0.05])).astype(np.float32)


def ids(y, k=0, p=1.0, m=0.0, invT=1.0):
    return SA.kept(np.asarray(y, dtype=np.float32), invT, k, p, m)[0].tolist()


def test_cuts_by_hand():
    assert ids(L) == [1, 3, 2, 0, 4] and ids(L, k=2) == [1, 3] and ids(L, k=9) == [1, 3, 2, 0, 4]
    assert ids(L, p=0.39) == [1] and ids(L, p=0.41) == [1, 3] and ids(L, p=0.66) == [1, 3, 2] and ids(L, p=0.96) == [1, 3, 2, 0, 4]
    assert ids(L, k=3, p=0.7) == [1, 3]              # 0.65 of 0.85 is over 0.7
    assert ids(L, m=0.3) == [1, 3, 2] and ids(L, m=0.7) == [1] and ids(L, m=1.0) == [1]
    assert ids(L, p=0.0) == ids(L, p=-1) == ids(L, m=2.0) == ids(L, k=1) == ids(L, p=math.nan) == ids(L, m=math.nan) == [1]
    assert ids(L, p=0.7, invT=4.0) == [1] and ids(L, p=0.7, invT=0.0) == [0, 1, 2, 3]  # sharper, and flat


def test_ties_and_values_that_take_no_part():
    assert ids(np.zeros(6), k=4) == [0, 1, 2, 3] and ids(np.zeros(6), p=0.5) == [0, 1, 2]
    assert ids([np.nan, 1.0, -np.inf, 1.0, np.nan], p=0.5) == [1] and ids([np.nan, -np.inf]) == []
    assert ids([0.0, np.inf, 1.0, np.inf], p=0.5) == [1]
    assert SA.choose(np.array([0.0, np.inf, np.inf], dtype=np.float32), np.zeros(3), 1.0, 0, 0.5, 0.0) == 1
    assert SA.choose(np.array([np.nan, np.nan], dtype=np.float32), np.zeros(2), 1.0, 0, 0.5, 0.0) == -1
    assert SA.choose(np.array([1.0, 3.0, 3.0], dtype=np.float32), None, 9.0, 1, 0.1, 0.5) == 1  # greedy


def test_against_brute_force():
    """The kept set is the smallest prefix of the order that the three rules allow."""
    rng = np.random.default_rng(0)
    for k, p, m in itertools.product((0, 1, 3, 7), (1.0, 0.9, 0.5, 0.1), (0.0, 0.05, 0.6)):
        y = rng.normal(0, 2, 9).astype(np.float32)
        order = sorted(range(9), key=lambda j: (-y[j], j))[: k or 9]
        w = [math.exp(float(y[j]) - float(y[order[0]])) for j in order]
        n = next((n for n in range(1, len(order) + 1) if sum(w[:n]) >= p * sum(w)), len(order)) if p < 1 else len(order)
        assert ids(y, k, p, m) == [j for i, j in enumerate(order[:n]) if i == 0 or w[i] >= m]


def test_frequencies_are_the_cut_distribution():
    rng = np.random.default_rng(1)
    got = np.zeros(5)
    for _ in range(20000):
        got[SA.choose(L, rng.gumbel(size=5), 1.0, 4, 0.9, 0.0)] += 1
    want = np.array([0.1, 0.4, 0.2, 0.25, 0]) / 0.95  # (0.85 of the first four's 0.95 is below 0.9: the fourth is kept too)
    chi = ((got[:4] - 20000 * want[:4]) ** 2 / (20000 * want[:4])).sum()
    assert got[4] == 0 and chi < 20


@pytest.mark.parametrize("noise", [True, False])
def test_without_cuts_the_walk_is_the_rules_walk(noise):
    rng = np.random.default_rng(2)
    for seed in range(20):
        logits, g = rng.normal(0, 1, (6, 12)).astype(np.float32), rng.gumbel(size=(4, 12)).astype(np.float32)
        tok, par = rng.integers(0, 12, 6), np.array([-1, 0, 0, 1, 1, 3])
        gn = (lambda k: g[k]) if noise else None
        word = rng.integers(0, 3, 12).astype(np.uint16)
        rest = dict(word=word, r=1.2, f=0.3, q=0.1, bias=[(3, 1.0)])
        assert SA.walk(lambda u: logits[u], gn, 0.8, 0, 1.0, 0.0, tok, par, 6, 3, **rest) == \
            RU.walk(lambda u: logits[u], gn, 0.8, tok, par, 6, 3, **rest)
