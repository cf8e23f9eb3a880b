"""Oracle for the acceptance walk under sampling rules (test infrastructure
only).

The walk is ``accept``'s (Sections 1 and 3: the policy's own choice at every
node); the policy's choice is made under the request's rules.  For token j, with
n the times j was said in the output so far, on this walk included, and p
whether the prompt holds it, every operation rounded to fp32:

    y = l;  if p or n > 0: y = y / r if y > 0 else y * r
    y = y - fl(f * n);  if n > 0: y = y - q
    y = y + each bias of j, in the order of the list
    x = y, or fl(fl(y * invT) + g)

over the tokens that the mask allows; a NaN or -inf is never chosen, ties go to
the lowest id, and where nothing is left the walk ends without a token.
A count word holds p in bit 15 and n (up to 32767) in the bits below.
"""
from __future__ import annotations

import numpy as np

F = np.float32


def scores(logits, noise, invT, word, said, r, f, q, bias, allowed):
    """fp32 [V]: x of every token, NaN where it cannot be chosen.

    word: uint16 [V] or None; said: tokens emitted on this walk; bias: list of
    (token, value); allowed: bool [V] or None."""
    y = np.array(logits, dtype=F)
    V = len(y)
    n = np.zeros(V, dtype=np.int64) if word is None else (word & 0x7FFF).astype(np.int64)
    p = np.zeros(V, dtype=bool) if word is None else (word & 0x8000) != 0
    for t in said:
        n[t] += 1
    with np.errstate(all="ignore"):
        held = p | (n > 0)
        y = np.where(held, np.where(y > 0, (y / F(r)).astype(F), (y * F(r)).astype(F)), y)
        y = (y - (F(f) * n.astype(F)).astype(F)).astype(F)
        y = np.where(n > 0, (y - F(q)).astype(F), y)
        for t, v in bias:
            if 0 <= t < V:
                y[t] = F(y[t] + F(v))
        if noise is not None:
            y = ((y * F(invT)).astype(F) + np.asarray(noise, dtype=F)).astype(F)
    y = np.where(np.isneginf(y), F(np.nan), y)
    return y if allowed is None else np.where(allowed, y, F(np.nan))


def allowed_of(mask_row, V: int) -> np.ndarray:
    """bool [V] of a row of 32-bit words, bit j % 32 of word j / 32."""
    w = np.asarray(mask_row).astype(np.int64) & 0xFFFFFFFF
    j = np.arange(V)
    return (w[j // 32] >> (j % 32)) & 1 == 1


def walk(row, noise, invT, tree_tokens, tree_parent, n_nodes: int, max_depth: int, word=None, r=1.0, f=0.0, q=0.0,
         bias=(), mask=None):
    """(n_accepted, out_tokens, out_nodes, n_emitted) of one sequence; row(u),
    noise(k) (or None) and mask(u) (or None) give rows."""
    u, k, tokens, nodes = 0, 0, [], []
    while True:
        logits = np.asarray(row(u), dtype=F)
        ok = None if mask is None else allowed_of(mask(u), len(logits))
        x = scores(logits, None if noise is None else noise(k), invT, word, tokens, r, f, q, bias, ok)
        if np.isnan(x).all():
            return k, tokens + [-1], nodes, k
        tok = int(np.nanargmax(x))
        kids = [c for c in range(u + 1, n_nodes) if tree_parent[c] == u and tree_tokens[c] == tok]
        tokens.append(tok)
        if not kids or k >= max_depth:
            return k, tokens, nodes, k + 1
        nodes.append(kids[0])
        u, k = kids[0], k + 1


def seen_add(word, tokens, prompt: bool, reset: bool):
    """The count row (uint16 [V]) after ``tokens`` have been entered."""
    w = np.zeros_like(word) if reset else word.copy()
    for t in tokens:
        if 0 <= t < len(w):
            if prompt:
                w[t] |= 0x8000
            elif w[t] & 0x7FFF < 0x7FFF:
                w[t] += 1
    return w
