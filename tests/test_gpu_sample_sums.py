"""The sums that the place of a top-p cut hangs on: how near the cut is to that of
exact sums, that it is the same one every time, and the counted tokens' part of them.

How far a sum may be off.  A weight is 2 ** x in fp32 with x = (z - M) log2(e) rounded:
half a unit in the last place of x, which is 2 ** -21 for |x| in [8, 16) and 2 ** -20 for
[16, 32), and log2(e) itself, off by 2 ** -26 of x, so by at most 2 ** -20 + 32 * 2 ** -26 =
1.5 * 2 ** -20 in x, times log(2) in the weight: 1.0e-6; the power function's unit in the last
place 2 ** -23; sums of up to 16 weights in fp32, 15 * 2 ** -24 = 0.9e-6.  A weight below
2 ** -32 of the largest is of no account.  Two more powers of that kind join the threads' sums
of the whole row (2 * (1.0e-6 + 2 ** -23 + 2 ** -24)).  So a part of the row is within 2.1e-6 of
what it weighs, the whole row within 4.6e-6, and the place of the cut is off by at most
6.7e-6 of the row's mass: BOUND."""
import math

import numpy as np
import pytest
import torch

from paper_2601_09083_amd import srt
from tests.test_gpu_sample import Case

pytestmark = pytest.mark.gpu
BOUND = 6.7e-6


def f32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32), device="cuda")


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")


def walk(z, noise, p, rules=None):
    """The token chosen at the root of each of B one-node trees, z [B, V]."""
    B = len(z)
    tree = (i32(np.zeros((B, 1))), i32(np.full((B, 1), -1)), i32(np.ones(B)))
    run = lambda: srt.srt_accept_sample(f32(z)[:, None], f32(noise)[:, None], srt.Sampling(top_p=f32(p)), *tree, 0, rules=rules)
    return run


@pytest.mark.parametrize("V,far", [(1 << 21, 13.015625), (1 << 21, 8.5), (262144, 12.0), (40001, 9.0), (5000, 3.3)])
def test_the_cut_inside_a_tail_of_ties(V, far):
    """One token of the largest score, all others at one distance from it: the kept ones are the first
    e of the row, up to BOUND.  Noise puts tokens further on than that first, three of them, then one
    before, which has to be the choice."""
    M = np.float32(9.625)
    z = np.full((5, V), M - np.float32(far), dtype=np.float32)
    noise = np.zeros((5, V), dtype=np.float32)
    w = math.exp(float(z[0, 0]) - float(M))
    mass = 1 + (V - 1) * w
    want = []
    for b, p in enumerate(np.array([0.3, 0.5, 0.8, 0.95, 0.999], dtype=np.float32)):
        z[b, V // 3] = M  # the first of the order; the others follow by their index
        e = math.ceil((float(p) * mass - 1) / w) if float(p) * mass > 1 else 0  # ties before which less than p of the mass lies
        off = math.ceil(BOUND * mass / w) + 2
        index = lambda i: i if i < V // 3 else i + 1  # of the i-th of the ties
        if e - off - 1 < 0:
            want.append(V // 3)
        else:
            want.append(index(e - off - 1))
            noise[b, want[-1]] = 4000.0
        for i, up in ((e + off, 5000.0), (e + 2 * off + 7, 7000.0), (e + 3 * off + 700, 6000.0)):
            if i < V - 1:
                noise[b, index(i)] = up
        noise[b, V // 3] = 1000.0
    got = walk(z, noise, np.array([0.3, 0.5, 0.8, 0.95, 0.999]))()
    assert got["out_tokens"][:, 0].tolist() == want


def test_the_cut_does_not_depend_on_the_order_of_atomics():
    """4000 counted tokens, which are listed in the order in which their waves come, weigh nearly all of
    the row; the cut lies in a tail of tokens of a billionth of the mass each, the last kept one of which
    the noise chooses."""
    V, said, B = 1 << 18, 4000, 8
    rng = np.random.default_rng(3)
    z = np.full((B, V), -10.6, dtype=np.float32)
    seen = np.zeros((B, V), dtype=np.int16)
    noise = np.broadcast_to(np.float32(64) + np.arange(V, dtype=np.float32) * np.float32(2.0 ** -13), (B, V)).copy()
    for b in range(B):
        t = rng.choice(V, said, replace=False)
        z[b, t] = rng.random(said) * 3.3 + 0.25
        seen[b, t] = 1
        noise[b, t] = 0
    rules = srt.Rules(seen=torch.as_tensor(seen, device="cuda"), frequency=f32([0.25] * B))
    y = np.where(seen > 0, z - np.float32(0.25), z).astype(np.float64)
    w = np.exp(y - y.max(1, keepdims=True))
    p = np.float32(1) - np.float32(2) ** -13
    run = walk(z, noise, [p] * B, rules)
    first = run()["out_tokens"][:, 0].clone()
    for b, tok in enumerate(first.tolist()):  # the ties up to the chosen one, and the counted ones before them all
        ties = seen[b] == 0
        before = w[b][~ties].sum() + w[b][ties][0] * ties[:tok].sum()
        assert abs(before - float(p) * w[b].sum()) <= BOUND * w[b].sum(), b
    for _ in range(12):
        assert torch.equal(run()["out_tokens"][:, 0], first)


@pytest.mark.parametrize("V", [3, 70, 4096, 4099, 16389, 40003, 262144])
def test_counted_tokens_wherever_they_lie(V):
    """None to more than are listed apart (4096), at a row's start, at its end and spread over it."""
    c = Case(31, 12, 3, V, 2, ruled=True, bias=4, cuts=[(0, 0.9, 0.0), (40, 1.0, 0.0), (0, 1.0, 0.05), (200, 0.9, 0.0)])
    rng = np.random.default_rng(V)
    c.words[:] = 0
    for b in range(c.B):
        n = min((0, 1, 4095, 4096, 4097, V // 2)[b // 2], V)
        t = np.arange(n) if b % 4 == 0 else np.arange(V - n, V) if b % 4 == 1 else rng.choice(V, n, replace=False)
        c.words[b, t] = rng.integers(1, 9, n)
    c.r[:], c.f[:], c.q[:] = 1.3, 0.2, 0.5
    c.check(c.run())
