"""Pins of the oracles of the 8-bit cache and of the sampling rules: closed
forms, library routines and brute force (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import accept as AC
from oracle import kv_quant as KQ
from oracle import rules as RU


def test_e4m3_table_is_the_librarys():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(KQ.e4m3_values(), want, equal_nan=True)


def test_e4m3_nearest_is_the_librarys_rounding():
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-448, 448, 20000), rng.normal(0, 0.01, 20000), rng.normal(0, 2 ** -8, 5000)])
    pos = KQ.e4m3_values()[:127]
    y = np.concatenate([y, (pos[1:] + pos[:-1]) / 2, -(pos[1:] + pos[:-1]) / 2, pos, -pos[1:]]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(KQ.e4m3_nearest(y), want)


@pytest.mark.parametrize("kv,half", [("e4m3", 2.0 ** -4), ("int8", None)])
def test_values_are_within_half_a_step(kv, half):
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.normal(0, 3, (16, 64)).astype(np.float32)).to(torch.bfloat16).float().numpy()
    codes, scale = KQ.quantise(x, kv)
    got = KQ.values(codes, kv) * float(scale)
    amp = np.abs(x).max()
    # e4m3: half a step relative, or half of the least subnormal step; int8: half a step of the page
    tol = np.maximum(half * np.abs(x), 2.0 ** -10 * amp / 448) if half else np.full_like(x, 0.5 * amp / 127)
    assert (np.abs(got - x) <= tol * (1 + 1e-5)).all()
    assert np.abs(got).max() == pytest.approx(amp, rel=1e-6)


def test_context_does_not_depend_on_arrival_and_keeps_the_open_page():
    rng = np.random.default_rng(2)
    rows = torch.from_numpy(rng.normal(0, 1, (37, 2, 8)).astype(np.float32)).to(torch.bfloat16).float().numpy()
    for kv in ("e4m3", "int8"):
        whole, codes, scales = KQ.context(rows, kv, 16)
        part, c2, s2 = KQ.context(rows[:33], kv, 16)
        assert np.array_equal(whole[:32], part[:32]) and np.array_equal(codes, c2) and np.array_equal(scales, s2)
        assert np.array_equal(whole[32:], rows[32:].astype(np.float64))


def test_zero_page_has_the_least_scale():
    for kv in ("e4m3", "int8"):
        codes, scale = KQ.quantise(np.zeros((16, 8), np.float32), kv)
        assert not codes.any() and scale == np.float32(2.0 ** -60 / KQ.TOP[kv])


def _tree(rng, N, V):
    par = [-1] + [int(rng.integers(0, i)) for i in range(1, N)]
    return rng.integers(0, V, N).tolist(), par


def test_walk_without_rules_is_the_plain_walk():
    rng = np.random.default_rng(3)
    for _ in range(30):
        N, V = 12, 7
        tok, par = _tree(rng, N, V)
        logits = rng.normal(0, 1, (N, V)).astype(np.float32)
        g = rng.gumbel(size=(6, V)).astype(np.float32)
        want = AC.accept(lambda u: logits[u], lambda k: g[k], 0.7, tok, par, N, 5)
        got = RU.walk(lambda u: logits[u], lambda k: g[k], 0.7, tok, par, N, 5)
        assert got == (*want, want[0] + 1)


def test_scores_by_hand():
    word = np.array([0, 2, 0x8000, 0x8001, 0], dtype=np.uint16)
    y = RU.scores([1, 3, -2, 4, -1], None, 1.0, word, [0, 1], 2.0, 0.5, 0.25, [(4, 1.5), (4, 0.25), (9, 7.0)], None)
    # 0: said once now: 1/2 - .5 - .25; 1: 3 times: 1.5 - 1.5 - .25; 2: prompt only: -4; 3: 2 - .5 - .25; 4: bias
    assert y.tolist() == [-0.25, -0.25, -4.0, 1.25, 0.75]


def test_masked_row_and_nothing_left():
    mask = np.array([0b101], dtype=np.uint32)
    assert RU.allowed_of(mask, 5).tolist() == [True, False, True, False, False]
    big = [float("nan"), float("inf"), -1.0]
    assert RU.walk(lambda u: big, None, 1.0, [5], [-1], 1, 3, mask=lambda u: np.array([0b100])) == (0, [2], [], 1)
    assert RU.walk(lambda u: big, None, 1.0, [5], [-1], 1, 3, mask=lambda u: np.array([0])) == (0, [-1], [], 0)
    low = [float("-inf")] * 3
    assert RU.walk(lambda u: low, None, 1.0, [5], [-1], 1, 3) == (0, [-1], [], 0)


def test_penalty_counts_the_walks_own_tokens():
    # a tree that repeats token 1; the second time its penalty lets token 0 win
    logits = [[1.0, 1.5]] * 3
    got = RU.walk(lambda u: logits[u], None, 1.0, [9, 1, 1], [-1, 0, 1], 3, 4, f=0.6)
    assert got == (1, [1, 0], [1], 2)


def test_seen_add():
    w = np.array([0, 0x7FFE, 0x8003, 5], dtype=np.uint16)
    got = RU.seen_add(w, [1, 1, 1, 2, 7, -1], False, False)
    assert got.tolist() == [0, 0x7FFF, 0x8004, 5]
    assert RU.seen_add(w, [3, 3], True, False).tolist() == [0, 0x7FFE, 0x8003, 0x8005]
    assert RU.seen_add(w, [3, 3], False, True).tolist() == [0, 0, 0, 2]
