"""Oracle of rows held in 8 bits (test infrastructure only, see the package docstring).

A row x of bf16 numbers is held as e4m3 codes and a power of two: e = the smallest integer >= -126
with max|x| <= 448 * 2^e over the finite elements, code = the e4m3 number nearest to x * 2^-e (ties
to the code with an even last bit), value = code * 2^e.  What is not finite becomes NaN.

The codes are looked up in the table of all e4m3 numbers; nothing here rounds by arithmetic.
"""
import math

import numpy as np

from .attention import widen_bf16

# the 127 finite magnitudes by code 0..126: exponent field f, three fraction bits
_GRID = np.array([(m / 8.0) * 2.0 ** -6 if f == 0 else (1 + m / 8.0) * 2.0 ** (f - 7)
                  for f in range(16) for m in range(8)][:127])
_MIDDLE = (_GRID[1:] + _GRID[:-1]) / 2          # exact: between codes i and i+1


def row_exponent(row):
    """row: float64 [256]."""
    finite = np.abs(row[np.isfinite(row)])
    top = float(finite.max()) if finite.size else 0.0
    e = -126
    if top > 0:
        e = math.frexp(top)[1] - 10              # below every candidate
        while top > math.ldexp(448.0, e):
            e += 1
    return max(e, -126)


def nearest_code(y):
    """Codes of magnitudes y (float64, at most 448)."""
    code = np.searchsorted(_MIDDLE, y, side="left")        # a tie goes to the lower code ..
    tie = np.isin(y, _MIDDLE)
    return np.where(tie & (code % 2 == 1), code + 1, code)  # .. unless that one is odd


def cached_values(bits):
    """What a cache in 8 bits holds for bf16 bit patterns [n, 256]: float64 [n, 256]."""
    x = widen_bf16(bits)
    out = np.empty_like(x)
    for i, row in enumerate(x):
        e = row_exponent(row)
        with np.errstate(invalid="ignore"):
            y = np.where(np.isfinite(row), np.abs(row), 0.0) * 2.0 ** -e
        value = np.ldexp(_GRID[nearest_code(y)], e)
        out[i] = np.where(np.isfinite(row), np.copysign(value, row), np.nan)
    return out


def bf16_bits(x):
    """Bit patterns of float64 numbers that are bf16 numbers (NaN: 0x7fc0; 2^128: infinity)."""
    with np.errstate(invalid="ignore", over="ignore"):
        u = np.asarray(x, dtype=np.float32).view(np.uint32)
    exact = (u & 0xffff) == 0
    assert np.all(exact | np.isnan(x)), "not a bf16 number"
    return np.where(np.isnan(x), 0x7fc0, u >> 16).astype(np.uint16)


def cached_source(source):
    """A data source whose keys and values are what a cache in 8 bits holds of `source`'s."""
    def read(recipe, layer, what, n):
        rows = source(recipe, layer, what, n)
        return rows if what == "q" else bf16_bits(cached_values(rows))
    return read
