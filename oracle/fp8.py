"""Oracle 8-bit floating point: blocks of 128 columns of 1 or 128 rows, one power of two each.

TEST INFRASTRUCTURE ONLY (see the package docstring).

For a block with largest finite magnitude A: s is the least integer >= -127 with
A <= 448 2^s; a code is the nearest e4m3 number to x / 2^s (ties to the even
code), found in the list of all of them; the exponent byte is s + 127.  Infinities
and NaN have the NaN code.  Values stay below 2^128, the end of fp32: with s = 120
numbers stop at 240.  Arrays: codes [rows, cols up to 16], bytes
[blocks of columns, blocks of rows up to 16].
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128
NAN = 0x7F


def numbers() -> np.ndarray:
    """The numbers of the codes 0 .. 126, ascending (sign 0)."""
    out = []
    for c in range(127):
        e, f = c >> 3, c & 7
        out.append(math.ldexp(f, -9) if e == 0 else math.ldexp(8 + f, e - 10))
    return np.array(out)


def exponent(top: float) -> int:
    s = -127
    while top > 448.0 * math.ldexp(1.0, s):
        s += 1
    return s + 127


def _codes(v: np.ndarray) -> np.ndarray:
    """The codes of the numbers nearest to v (finite, |v| <= 448)."""
    table = numbers()
    a = np.abs(v)
    hi = np.searchsorted(table, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = table[hi] - a, a - table[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (c | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def pack(x, block_rows=1):
    rows, cols = x.shape
    nb, nr = -(-cols // BLOCK), -(-rows // block_rows)
    code = np.zeros((rows, -(-cols // 16) * 16), np.uint8)
    exp = np.zeros((nb, -(-nr // 16) * 16), np.uint8)
    for b in range(nb):
        at = slice(b * BLOCK, min(cols, (b + 1) * BLOCK))
        part = x[:, at]
        fine = np.isfinite(part)
        top = np.where(fine, np.abs(part), 0).max(1)
        for r in range(nr):
            exp[b, r] = exponent(float(top[r * block_rows:(r + 1) * block_rows].max()))
        e = np.repeat(exp[b, :nr], block_rows)[:rows].astype(np.int64)[:, None]
        with np.errstate(all="ignore"):
            v = np.where(fine, part, 0) * np.ldexp(1.0, 127 - e)
        v = np.where(e == 247, np.clip(v, -240, 240), v)
        code[:, at] = np.where(fine, _codes(v), NAN)
    return code, exp


def unpack(code, exp, cols, block_rows=1):
    rows = len(code)
    table = numbers()
    c = code[:, :cols]
    v = np.where((c & 127) == NAN, np.nan, table[np.minimum(c & 127, 126)]) * np.where(c >= 128, -1.0, 1.0)
    e = np.repeat(exp.T.astype(np.int64), block_rows, 0)[:rows]
    s = np.where(e == 255, np.nan, np.ldexp(1.0, e - 127))
    return v * np.repeat(s, BLOCK, 1)[:, :cols]
