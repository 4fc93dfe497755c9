"""8-bit activation checkpoints from their definition, in float64.

Each row is cut into groups of 32 columns (the last may be shorter).  With qmax
= 127 (int8) or 448 (e4m3), k is the smallest integer >= -126 with max |x| <=
qmax 2^k; an element is held as x / 2^k rounded to the format (nearest, ties to
even), the group by the byte k + 127.  A group with a value that is not finite
reads back as NaN (byte 255).

TEST INFRASTRUCTURE ONLY.
"""

from __future__ import annotations

import numpy as np

GROUP = 32
QMAX = {"int8": 127.0, "e4m3": 448.0}
# the non-negative e4m3 values in order: their index is their bit pattern
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] +
                [(8 + m) / 8.0 * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)])


def _nearest_e4m3(v):
    a = np.abs(v)
    hi = np.clip(np.searchsorted(E4M3, a), 1, len(E4M3) - 1)
    lo = hi - 1
    down, up = a - E4M3[lo], E4M3[hi] - a
    idx = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.copysign(E4M3[idx], v)


def pack(x, fmt):
    """(values, bytes): what a checkpoint of x [rows, cols] stands for, and its
    scale bytes [rows, ceil(cols / 32)]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    n = -(-cols // GROUP)
    vals, scales = np.empty_like(x), np.zeros((rows, n), dtype=np.uint8)
    for g in range(n):
        part = x[:, g * GROUP:(g + 1) * GROUP]
        finite = np.all(np.isfinite(part), axis=1)
        top = np.where(finite, np.max(np.abs(np.where(np.isfinite(part), part, 0.0)), axis=1, initial=0.0), 0.0)
        k = np.full(rows, -126)
        while np.any(bad := top > QMAX[fmt] * np.exp2(k.astype(np.float64))):
            k[bad] += 1
        scaled = np.where(finite[:, None], part, 0.0) / np.exp2(k.astype(np.float64))[:, None]
        q = np.rint(scaled) if fmt == "int8" else _nearest_e4m3(scaled)
        q = q * np.exp2(k.astype(np.float64))[:, None]
        vals[:, g * GROUP:(g + 1) * GROUP] = np.where(finite[:, None], q, np.nan)
        scales[:, g] = np.where(finite, k + 127, 255)
    return vals, scales
