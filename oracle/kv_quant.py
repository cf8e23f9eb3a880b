"""Oracle for the KV cache held in 8 bits (test infrastructure only).

The paper keeps the policy's KV cache in the engine's format (Appendix C only
asks that one pass reads it once); this is the format of a cache held in 8 bits
with a scale for each page of tokens and KV head.  A full page of one head and
tensor, x [page, d], is stored as

    amp = max(max |x|, 2^-60), top = 448 (e4m3) or 127 (int8)
    scale = fl32(amp / top)
    code = nearest code, ties to even, of min(max(fl32(x * fl32(top / amp)), -top), top)

and stands for code * scale; the positions of the page that is not full yet
keep their bf16 vectors.  The context is a function of the tokens alone, so
this module computes it from the whole history of a sequence at once.

e4m3 is written out from its definition: sign, 4 exponent bits with bias 7, 3
mantissa bits, exponent field 0 subnormal, no infinities, all ones NaN.
"""
from __future__ import annotations

import numpy as np

TOP = {"e4m3": 448.0, "int8": 127.0}
LEAST_AMP = 2.0 ** -60


def e4m3_values() -> np.ndarray:
    """The 256 values of the codes, float64 (NaN at 0x7f and 0xff)."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = (m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            x = np.nan
        v[c] = -x if c & 128 else x
    return v


_VALUES = e4m3_values()
_POSITIVE = _VALUES[:127]  # 0 .. 448, ascending; code = index


def e4m3_nearest(y: np.ndarray) -> np.ndarray:
    """Codes nearest to y (|y| <= 448), ties to the even code."""
    a = np.abs(np.asarray(y, dtype=np.float64))
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)  # first value >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code + np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantise(x: np.ndarray, kv: str):
    """x [page, d] float32 -> (codes uint8 or int8 [page, d], scale float32)."""
    x = np.asarray(x, dtype=np.float32)
    top = np.float32(TOP[kv])
    amp = np.float32(max(float(np.abs(x).max()), LEAST_AMP))
    y = np.clip((x * (top / amp).astype(np.float32)).astype(np.float32), -top, top)
    codes = e4m3_nearest(y) if kv == "e4m3" else np.rint(y).astype(np.int8)
    return codes, np.float32(amp / top)


def values(codes: np.ndarray, kv: str) -> np.ndarray:
    """float64 values of codes before the scale."""
    return _VALUES[np.asarray(codes).view(np.uint8)] if kv == "e4m3" else np.asarray(codes).astype(np.float64)


def context(rows: np.ndarray, kv: str, page: int):
    """rows [L, Hkv, d] float32 (the bf16 vectors of all tokens so far) ->
    (values float64 [L, Hkv, d], codes and scales of the full pages
    [pages, Hkv, page, d] / [pages, Hkv])."""
    L, H, d = rows.shape
    full = L // page
    out = np.array(rows, dtype=np.float64)
    codes = np.zeros((full, H, page, d), dtype=np.uint8 if kv == "e4m3" else np.int8)
    scales = np.zeros((full, H), dtype=np.float32)
    for i in range(full):
        for h in range(H):
            c, s = quantise(rows[i * page:(i + 1) * page, h], kv)
            codes[i, h], scales[i, h] = c, s
            out[i * page:(i + 1) * page, h] = values(c, kv) * np.float64(s)
    return out, codes, scales
