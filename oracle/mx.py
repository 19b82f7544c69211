"""Blocks of 32 elements with a shared power-of-two scale, in fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A code is looked up in the table of its format's values: e2m1 (1 sign, 2 exponent and 1 fraction bit) and e4m3
(1, 4, 3; the all-ones code is NaN and never written). The scale exponent of a block is the smallest e at which the
block's largest magnitude is at most T 2^e, held to [lowest, 127 - emax], where T is the midpoint between the largest
code and the next step above it (7 for e2m1, 464 for e4m3): at most that far the largest code is a nearest one.
"""

from __future__ import annotations

import numpy as np

BLOCK = 32
#            values of the non-negative codes in order, T, largest code's exponent, lowest scale exponent
_E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
_E4M3 = np.array([np.ldexp(m if e == 0 else 8 + m, max(e, 1) - 10) for e in range(16) for m in range(8)][:127])
FORMATS = {"mxfp4": (_E2M1, 7.0, 2, -127), "mxfp8": (_E4M3, 464.0, 8, -124)}


def quantise(x, fmt):
    """(code numbers with sign bit, scale bytes) of ``x`` [..., d]."""
    table, most, emax, lowest = FORMATS[fmt]
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(*x.shape[:-1], -1, BLOCK)
    amax = np.abs(y).max(-1)
    bad = ~np.isfinite(amax)
    m, p = np.frexp(np.where(bad, 1.0, amax) / most)  # amax / T = m 2^p with m in [0.5, 1)
    e = np.where(amax == 0, lowest, np.where(m == 0.5, p - 1, p))
    e = np.clip(e, lowest, 127 - emax)
    mag = np.abs(np.where(bad[..., None], 0.0, y)) * np.ldexp(1.0, -e)[..., None]
    mids = (table[1:] + table[:-1]) / 2
    down, up = np.searchsorted(mids, mag, "left"), np.searchsorted(mids, mag, "right")
    code = np.where(down % 2 == 0, down, up)  # they differ on a tie: the even code
    sign = np.signbit(np.where(bad[..., None], 0.0, y)).astype(code.dtype)
    code = code + sign * (8 if fmt == "mxfp4" else 128)
    return code.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def pack(code, fmt):
    """Bytes of code numbers [..., d]."""
    if fmt == "mxfp8":
        return code.astype(np.uint8)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def values(codes, scales, fmt):
    """What bytes of codes and scales stand for."""
    table = FORMATS[fmt][0]
    c = codes.astype(np.int64)
    if fmt == "mxfp4":
        c = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)
    half = 8 if fmt == "mxfp4" else 128
    table = np.append(table, np.nan) if fmt == "mxfp8" else table
    v = np.where(c >= half, -table[c % half], table[c % half])
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, -1)
