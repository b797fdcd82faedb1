"""Oracle: rotary embedding in its layouts and scalings, rows by slot (float64).

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

Pair i < R / 2 of a head's first R values turns by p * f_i; the pair is elements
(i, i + R / 2) ("half") or (2 i, 2 i + 1) ("interleaved").  With w_i = base**(-2 i /
R): f_i = w_i; "linear" w_i / s; "parts" (YaRN, Sec. 3.2) w_i (c + (1 - c) / s), c the
place of r_i = L w_i / (2 pi) between alpha and beta; "yarn" the same with c falling
linearly in i between the pairs that turn beta and alpha times over L.

Pins: ``tests/test_oracle_rotary.py``.
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(R, base, scaling=None, factor=1.0, orig_ctx=0.0, alpha=0.0, beta=0.0):
    out = []
    for i in range(R // 2):
        w = base ** (-2.0 * i / R)
        if scaling is None:
            out.append(w)
        elif scaling == "linear":
            out.append(w / factor)
        else:
            if scaling == "parts":
                c = (orig_ctx * w / (2 * math.pi) - alpha) / (beta - alpha)
            else:
                def pair(x):    # w_i = 2 pi x / L  <=>  i = (R / 2) log_base(L / (2 pi x))
                    return R / 2 * math.log(orig_ctx / (2 * math.pi * x)) / math.log(base)
                lo, hi = max(math.floor(pair(beta)), 0), min(math.ceil(pair(alpha)), R - 1)
                c = 1 - (i - lo) / max(hi - lo, 0.001)
            c = min(max(c, 0.0), 1.0)
            out.append(w * (c + (1 - c) / factor))
    return np.array(out)


def rotate(x, pos, freqs, layout="half", mscale=1.0, sections=None):
    """x [N][H][D]; pos [N], or [3][N] with sections."""
    x = np.array(x, dtype=np.float64)
    h = len(freqs)
    pos = np.asarray(pos, dtype=np.float64)
    for i in range(h):
        axis = 0 if sections is None else 0 if i < sections[0] else 1 if i < sections[0] + sections[1] else 2
        p = pos if sections is None else pos[axis]
        a, b = (i, i + h) if layout == "half" else (2 * i, 2 * i + 1)
        z = (x[..., a] + 1j * x[..., b]) * (mscale * np.exp(1j * p * freqs[i]))[:, None]
        x[..., a], x[..., b] = z.real, z.imag
    return x


def put_rows(cache, slots, rows):
    """Rows [N][H][D] into a copy of a cache [blocks][H][rows][D] at their slots (< 0: nowhere)."""
    out = np.array(cache)
    for n, s in enumerate(slots):
        if s >= 0:
            out[s // out.shape[2], :, s % out.shape[2]] = rows[n]
    return out
