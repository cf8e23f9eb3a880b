"""Pins of the rotary encoding's oracle: closed forms and invariants (no GPU)."""
import math

import numpy as np

from oracle import rope as RO

INV = np.array([1.0, 0.25, 2.0 ** -10, 0.0])


def test_by_hand():
    x = np.array([[3.0, 5.0, 1.0, 2.0, 4.0, 7.0, -1.0, 6.0, 9.0]])  # one head of 9 dims, 8 of which turn
    got = RO.turn(x, 2, INV, False, 1.0)[0]
    for m, a in enumerate((2.0, 0.5, 2.0 ** -9, 0.0)):
        x0, x1 = x[0, m], x[0, m + 4]
        assert math.isclose(got[m], x0 * math.cos(a) - x1 * math.sin(a), rel_tol=1e-14)
        assert math.isclose(got[m + 4], x1 * math.cos(a) + x0 * math.sin(a), rel_tol=1e-14)
    assert got[8] == 9.0
    got = RO.turn(x, 2, INV, True, 0.5)[0]
    for m, a in enumerate((2.0, 0.5, 2.0 ** -9, 0.0)):
        x0, x1 = x[0, 2 * m], x[0, 2 * m + 1]
        assert math.isclose(got[2 * m], 0.5 * (x0 * math.cos(a) - x1 * math.sin(a)), rel_tol=1e-14)
        assert math.isclose(got[2 * m + 1], 0.5 * (x1 * math.cos(a) + x0 * math.sin(a)), rel_tol=1e-14)


def test_products_depend_on_the_distance_alone():
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(2, 1, 8))
    for inter in (False, True):
        dot = lambda a, b: float((RO.turn(q, a, INV, inter, 1.0) * RO.turn(k, b, INV, inter, 1.0)).sum())
        assert math.isclose(dot(7, 3), dot(107, 103), rel_tol=1e-9)
        assert not math.isclose(dot(7, 3), dot(7, 4), rel_tol=1e-3)
        assert np.allclose(RO.turn(q, 0, INV, inter, 1.0), q)
        assert math.isclose(np.linalg.norm(RO.turn(q, 12345, INV, inter, 1.0)), np.linalg.norm(q), rel_tol=1e-12)


def test_places():
    row = [5, -1, 9, 0]
    assert RO.slot(row, 16, 9, 0) == (5, 0) and RO.slot(row, 16, 9, 63) == (0, 15)
    assert RO.slot(row, 16, 9, 16) is None and RO.slot(row, 16, 9, 32) is None  # no page; beyond the pool
    assert RO.slot(row, 16, 9, 64) is None and RO.slot(row, 16, 9, -1) is None
