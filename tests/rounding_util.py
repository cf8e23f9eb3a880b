"""Rows that the rounding of a score decides.

A score is a chain of fp32 operations, each rounded by itself.  One that takes a
product into the sum behind it without rounding it (a fused multiply-add) is off
by a last bit now and then.  Here a row's best token has such a score, and its
rival has the separately rounded value to the bit: behind the token where the
fused score is the smaller one, ahead of it where it is the larger, so that the
two ways of computing it give different tokens."""
from __future__ import annotations

import numpy as np

from oracle import rules as RU

F = np.float32
LOW = -60.0     # every other logit
FAR = 1000.0    # the token that leads to the row's node


def fma(a, b, c):
    """a * b + c rounded once: the product of two fp32 is exact in fp64."""
    return F(np.float64(a) * np.float64(b) + np.float64(c))


def to_bf16(x):
    u = np.array([x], dtype=F).view(np.uint32)
    return F((((u + 0x8000) >> 16) << 16).astype(np.uint32).view(F)[0])


class Planted:
    """B trees of a root and one child.  Odd sequences walk to the child and are
    decided there, even ones at the root.  ``kinds`` are taken in turn:

    * freq   y - frequency * count
    * rep    y * repetition - frequency * count, y negative
    * bias   the same as freq, for a token with a bias
    * path   the same as freq, for the token that the walk has just emitted (odd sequences)
    * noise  y * inv_temperature + gumbel, of an ordinary token
    * noise_bias, noise_path   the same of a token with a bias of zero, of the emitted token

    and the places too: in the row, in its last three entries (V % 4 is 3)."""

    def __init__(self, seed, B, V, kinds, sampled, bf16=False):
        assert V % 4 == 3
        rng = np.random.default_rng(seed)
        self.B, self.N, self.V, self.dmax, self.invT = B, 2, V, 1, F(0.9) if sampled else F(1.0)
        self.logits = np.full((B, 2, V), LOW, dtype=F)
        self.gumbel = np.zeros((B, 2, V), dtype=F) if sampled else None
        self.words = np.zeros((B, V), dtype=np.uint16)
        self.r, self.f, self.q = np.ones(B, F), np.zeros(B, F), np.zeros(B, F)
        self.bias = [[] for _ in range(B)]
        self.tok = np.full((B, 2), -1, dtype=np.int32)
        self.par = np.tile(np.array([-1, 0], np.int32), (B, 1))
        self.n = np.full(B, 2)
        self.fused = np.zeros(B, dtype=np.int64)   # the token that fused scores give
        for b in range(B):
            kind, u = kinds[(b // 2) % len(kinds)], b % 2
            if kind.endswith("path") and u == 0:
                kind = {"path": "freq", "noise_path": "noise"}[kind]
            last = (b // (2 * len(kinds))) % 2 == 1
            while True:
                c, f, r, v, g = int(rng.integers(1, 9)), F(rng.uniform(0.1, 2)), F(1), F(0), F(0)
                y = F(rng.uniform(0.5, 8))
                if kind == "rep":
                    y, r = F(-y), F(rng.uniform(1.05, 1.6))
                if kind == "bias":
                    v = F(rng.normal())
                if kind == "path" and rng.random() < 0.5:
                    c = 1  # nothing in the count row
                if kind.startswith("noise"):
                    f, g = F(0), F(rng.gumbel())
                    y = to_bf16(y) if bf16 else y
                z = F(y * r)
                one_by_one = F(F(z - F(f * F(c))) + v)
                other = [F(fma(-f, F(c), z) + v), F(fma(y, r, -F(f * F(c))) + v)]
                if kind.startswith("noise"):
                    one_by_one, other = F(F(y * self.invT) + g), [fma(y, self.invT, g)]
                elif kind != "rep":
                    other = other[:1]
                side = {bool(x < one_by_one) for x in other}
                if one_by_one not in other and len(side) == 1 and one_by_one != 0:
                    break
            behind = side.pop()
            if last:
                t, rival = (V - 2, V - 1) if behind else (V - 1, V - 3)
            else:
                t, rival = sorted(int(x) for x in rng.choice(V - 3, 2, replace=False))
                if not behind:
                    t, rival = rival, t
            self.fused[b] = rival if behind else t
            self.tok[b, 1] = t if kind.endswith("path") else int(rng.choice([x for x in (5, 6, 7) if x not in (t, rival)]))
            if u == 1:
                self.logits[b, 0, self.tok[b, 1]] = FAR
            self.logits[b, u, t] = y
            if sampled:
                self.gumbel[b, u, t], self.gumbel[b, u, rival] = g, one_by_one
                self.logits[b, u, rival] = 0
            else:
                self.logits[b, u, rival] = one_by_one
            if not kind.startswith("noise"):
                self.words[b, t] = c - (kind == "path")
                self.r[b], self.f[b] = r, f
            if kind == "noise_bias" or kind == "bias":
                self.bias[b] = [(t, float(v))]

    def want(self, b):
        """(n_accepted, out_tokens, out_nodes, n_emitted) of the oracle's walk."""
        return RU.walk(lambda u: self.logits[b, u], None if self.gumbel is None else lambda k: self.gumbel[b, k], self.invT,
                       self.tok[b], self.par[b], 2, self.dmax, self.words[b], self.r[b], self.f[b], self.q[b], self.bias[b])

    def check(self, got):
        toks = got["out_tokens"].cpu().numpy()
        fused = 0
        for b in range(self.B):
            k, t, _, _ = self.want(b)
            assert int(got["n_accepted"][b]) == k == b % 2, b
            fused += int(toks[b, k]) == self.fused[b]
        assert fused == 0, f"{fused} of {self.B} rows are decided by scores that lack a rounding"
        for b in range(self.B):
            k, t, _, _ = self.want(b)
            assert toks[b, :k + 1].tolist() == t, b


GREEDY = ("freq", "rep", "bias", "path")
SAMPLED = ("noise", "noise_bias", "noise_path")
