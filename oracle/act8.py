"""Oracle 8-bit activations: blocks of 32 columns with one power of two each.

TEST INFRASTRUCTURE ONLY (see the package docstring).

For a block with largest magnitude A: s is the least integer >= -127 with
A <= 127 2^s, a code is the nearest integer to x / 2^s (ties to even), and the
exponent byte is s + 127; a block of zeros has byte 0, one that holds an
infinity or a NaN has byte 255 (codes 0) and reads as NaN.  Values stay below
2^128, the end of fp32: with s = 122 codes stop at 63.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32


def exponent(top: float) -> int:
    """The byte of a block with largest magnitude `top`, by search."""
    if not math.isfinite(top):
        return 255
    s = -127
    while top > 127.0 * math.ldexp(1.0, s):
        s += 1
    return s + 127


def pack(x):
    """x [rows, cols] float64 -> (codes int8, bytes uint8 [rows, ceil(cols / 32)])."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    code = np.zeros((rows, cols), np.int8)
    exp = np.zeros((rows, nb), np.uint8)
    for b in range(nb):
        at = slice(b * BLOCK, min(cols, (b + 1) * BLOCK))
        top = np.abs(x[:, at]).max(1)
        top = np.where(np.isnan(x[:, at]).any(1), np.nan, top)
        e = np.array([exponent(float(t)) for t in top])
        exp[:, b] = e
        ok = e != 255
        with np.errstate(all="ignore"):
            v = np.rint(x[:, at] * np.ldexp(1.0, 127 - e)[:, None])
        v = np.where((e == 249)[:, None], np.clip(v, -63, 63), v)
        code[ok, at] = v[ok].astype(np.int8)
    return code, exp


def unpack(code, exp):
    scale = np.ldexp(1.0, exp.astype(np.int64) - 127)
    scale[exp == 255] = np.nan
    return code.astype(np.float64) * np.repeat(scale, BLOCK, 1)[:, :code.shape[1]]
