"""Oracle: rows of a 4-bit KV cache (float64).

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

A row x of D values is D / 32 blocks of 32 e2m1 codes (sign, 2 exponent bits of
bias 1, 1 mantissa bit) and one exponent byte e each; a block stands for ``code *
2**(e - 127)``.  e is the smallest integer in [1, 254] with max |x_i| <= 7 *
2**(e - 127), and a code the nearest value to x_i * 2**(127 - e), ties to the
even code, at most 6; a block that holds an infinity or NaN has e = 255 (32 NaN)
and codes 0.  Two codes share a byte, the first in its low half.  The paper does
not fix a cache's storage type.

Pins: ``tests/test_oracle_quant4.py``.
"""
from __future__ import annotations

import numpy as np


def code_values():
    """The 16 codes' values, from their bit fields."""
    out = np.empty(16)
    for c in range(16):
        sign, exp, man = c >> 3, (c >> 1) & 3, c & 1
        mag = 0.5 * man if exp == 0 else (1 + 0.5 * man) * 2.0 ** (exp - 1)
        out[c] = -mag if sign else mag
    return out


_VALUES = code_values()


def nearest_code(x):
    """Codes of values |x| <= 7, to nearest, ties to the even code (by search)."""
    x = np.asarray(x, dtype=np.float64)
    d = np.abs(np.abs(x)[..., None] - _VALUES[:8])
    # of two that are equally near, the even one: odd codes count as a hair farther
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    c = order[d[..., order].argmin(axis=-1)]
    return (c + 8 * np.signbit(x)).astype(np.uint8)


def encode(x):
    """Rows x [..., D] as (codes [..., D], one a byte; exponents [..., D / 32])."""
    x = np.asarray(x, dtype=np.float64)
    x = x.reshape(x.shape[:-1] + (-1, 32))
    fine = np.isfinite(x).all(axis=-1)
    safe = np.where(fine[..., None], x, 0.0)
    top = np.abs(safe).max(axis=-1)
    e = np.ones(top.shape, dtype=np.int64)
    for k in range(1, 254):
        e += top > 7.0 * 2.0 ** (k - 127)
    c = nearest_code(safe * 2.0 ** (127.0 - e[..., None]))
    c = np.where(fine[..., None], c, 0).reshape(c.shape[:-2] + (-1,))
    return c.astype(np.uint8), np.where(fine, e, 255).astype(np.uint8)


def pack(codes):
    """Codes [..., D] as bytes [..., D / 2]."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(b):
    out = np.empty(b.shape[:-1] + (2 * b.shape[-1],), np.uint8)
    out[..., 0::2], out[..., 1::2] = b & 15, b >> 4
    return out


def decode(codes, exps):
    """The values [..., D] of codes [..., D] and exponents [..., D / 32]."""
    unit = np.where(exps == 255, np.nan, 2.0 ** (np.asarray(exps, dtype=np.float64) - 127.0))
    return _VALUES[codes] * np.repeat(unit, 32, axis=-1)
