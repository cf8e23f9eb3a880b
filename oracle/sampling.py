"""Oracle for the acceptance walk of a policy that samples with a temperature,
top-k, top-p and min-p (test infrastructure only).

The walk is ``rules``'s; the choice at a row, from its logits y under the rules (NaN
where a token cannot be chosen) and noise g:

    z = fl(y * invT); tokens in the order of z descending, id ascending;
    the first k of them (k <= 0: all); of these, those before which the mass
    exp(z - max z) is below p times the mass of all of these (p >= 1: all); of
    these, those with exp(z - max z) >= min_p (min_p <= 0: all); the first always;
    the largest fl(z + g) of what is kept, lowest id on ties.

Masses are fp64 sums.  Without noise the choice is the largest y.
"""
from __future__ import annotations

import math

import numpy as np

from . import rules as RU

F = np.float32


def kept(y, invT, k: int, p: float, min_p: float):
    """(ids that are kept, in order; z fp32 [V])."""
    with np.errstate(all="ignore"):
        z = (np.asarray(y, dtype=F) * F(invT)).astype(F)
    z = np.where(np.isnan(z), F(-np.inf), z)
    order = np.lexsort((np.arange(len(z)), -z.astype(np.float64)))
    order = order[z[order] > -np.inf]
    if not len(order):
        return order, z
    if k > 0:
        order = order[:k]
    with np.errstate(invalid="ignore"):
        d = z[order].astype(np.float64) - float(z[order[0]])
    w = np.exp(d, where=~np.isnan(d), out=np.ones(len(d)))
    before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
    keep = np.ones(len(order), dtype=bool)
    if not float(p) >= 1:
        keep &= before < float(p) * math.fsum(w)
    if not float(min_p) <= 0:
        keep &= d >= math.log(min_p) if min_p == min_p else False
    keep[0] = True
    return order[keep], z


def choose(y, noise, invT, k: int, p: float, min_p: float) -> int:
    """The chosen id, -1 if there is none."""
    if noise is None:
        y = np.where(np.isneginf(y), F(np.nan), y)
        return -1 if np.isnan(y).all() else int(np.nanargmax(y))
    ids, z = kept(y, invT, k, p, min_p)
    x = (z[ids] + np.asarray(noise, dtype=F)[ids]).astype(F)
    ok = ~np.isnan(x) & ~np.isneginf(x)
    if not ok.any():
        return -1
    return int(ids[ok][x[ok] == x[ok].max()].min())


def walk(row, noise, invT, k, p, min_p, tree_tokens, tree_parent, n_nodes: int, max_depth: int, word=None, r=1.0, f=0.0,
         q=0.0, bias=(), mask=None):
    """(n_accepted, out_tokens, out_nodes, n_emitted) of one sequence, as ``rules.walk``."""
    u, step, tokens, nodes = 0, 0, [], []
    while True:
        logits = np.asarray(row(u), dtype=F)
        ok = None if mask is None else RU.allowed_of(mask(u), len(logits))
        y = RU.scores(logits, None, 1.0, word, tokens, r, f, q, bias, ok)
        tok = choose(y, None if noise is None else noise(step), invT, k, p, min_p)
        if tok < 0:
            return step, tokens + [-1], nodes, step
        kids = [c for c in range(u + 1, n_nodes) if tree_parent[c] == u and tree_tokens[c] == tok]
        tokens.append(tok)
        if not kids or step >= max_depth:
            return step, tokens, nodes, step + 1
        nodes.append(kids[0])
        u, step = kids[0], step + 1
