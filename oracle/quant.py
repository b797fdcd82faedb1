"""Oracle: rows of an 8-bit KV cache (float64).

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

A row x of D values is D e4m3 codes (OCP 8-bit floats: sign, 4 exponent bits of
bias 7, 3 mantissa bits, no infinity, 0x7f and 0xff NaN, largest 448) and one
exponent byte e; it stands for ``code * 2**(e - 127)``.  e is the smallest
integer in [1, 254] with max |x_i| <= 448 * 2**(e - 127) over the finite x_i,
and a code the nearest value to x_i * 2**(127 - e), ties to the even code;
infinities and NaN become NaN.  The paper does not fix a cache's storage type;
8-bit rows halve the bytes that its verify step reads.

Pins: ``tests/test_oracle_quant.py``.
"""
from __future__ import annotations

import numpy as np


def code_values():
    """The 256 codes' values, from their bit fields."""
    out = np.empty(256)
    for c in range(256):
        sign, exp, man = c >> 7, (c >> 3) & 15, c & 7
        if exp == 15 and man == 7:
            out[c] = np.nan
            continue
        mag = (man / 8.0) * 2.0 ** -6 if exp == 0 else (1 + man / 8.0) * 2.0 ** (exp - 7)
        out[c] = -mag if sign else mag
    return out


_VALUES = code_values()
_MAGS = _VALUES[:127]                       # ascending: 0 .. 448


def nearest_code(x):
    """Codes (uint8) of values |x| <= 448, to nearest, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    hi = np.searchsorted(_MAGS, a, side="left").clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    dh, dl = _MAGS[hi] - a, a - _MAGS[lo]
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(hi % 2 == 0, hi, lo)))
    return (c + 128 * np.signbit(x)).astype(np.uint8)


def exponent(top):
    """The exponent byte of rows whose largest finite magnitude is ``top``."""
    out = np.ones(np.shape(top), dtype=np.int64)
    for e in range(1, 254):
        out += np.asarray(top, dtype=np.float64) > 448.0 * 2.0 ** (e - 127)
    return out


def encode(x):
    """Rows x [..., D] (float64 values) as (codes [..., D], exponents [...]), uint8."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    e = exponent(np.where(fine, np.abs(x), 0.0).max(axis=-1))
    codes = nearest_code(np.where(fine, x, 0.0) * 2.0 ** (127.0 - e[..., None]))
    return np.where(fine, codes, 0x7f).astype(np.uint8), e.astype(np.uint8)


def decode(codes, exps):
    """The values [..., D] that rows stand for."""
    return _VALUES[codes] * 2.0 ** (np.asarray(exps, dtype=np.float64)[..., None] - 127.0)


def bf16(x):
    """float64 -> float32 -> bf16, each to nearest, ties to even, as float64."""
    u = np.asarray(x, dtype=np.float64).astype(np.float32).view(np.uint32)
    r = (u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000
    return r.astype(np.uint32).view(np.float32).astype(np.float64)
