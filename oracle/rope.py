"""Oracle for the rotary position encoding and for where a step's keys and values
go (test infrastructure only).

The pair (x0, x1) m of a head at position p turns by the angle p * inv_freq[m]:
as a complex number it is multiplied by factor * e^(i angle).  A pair is the dims
m and m + rot / 2 of a head or, interleaved, 2 m and 2 m + 1; dims from rot on
stay.  Everything is fp64.
"""
from __future__ import annotations

import numpy as np


def turn(x, pos, inv_freq, interleaved: bool, factor: float):
    """x [..., heads, d] at positions pos [...] (fp64 in, fp64 out)."""
    x = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    m = np.arange(half)
    lo, hi = (2 * m, 2 * m + 1) if interleaved else (m, m + half)
    angle = np.asarray(pos, dtype=np.float64)[..., None] * np.asarray(inv_freq, dtype=np.float64)
    z = (x[..., lo] + 1j * x[..., hi]) * (factor * np.exp(1j * angle))[..., None, :]
    x[..., lo], x[..., hi] = z.real, z.imag
    return x


def slot(block_table_row, page: int, num_pages: int, position: int):
    """(page id, slot) of a position, or None where it has no place."""
    if position < 0 or position >= len(block_table_row) * page:
        return None
    pg = int(block_table_row[position // page])
    return (pg, position % page) if 0 <= pg < num_pages else None
