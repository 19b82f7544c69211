"""Rotary positions with several axes, in fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Pair i of a row is a complex number that is multiplied by exp(i phi), phi = pos[axis_i] * freq_i; elements
past the pairs stay. The inverse multiplies by the conjugate, which is also the transposed map: the gradient.
"""

from __future__ import annotations

import numpy as np


def rope(x, pos, freq, axis, pairing="interleaved", inverse=False):
    """``x`` [B, H, S, d], ``pos`` [S, A] or [B, S, A], ``freq`` and ``axis`` [n]."""
    x = np.asarray(x, dtype=np.float64)
    pos = np.asarray(pos, dtype=np.float64)
    if pos.ndim == 2:
        pos = pos[None]
    phi = (pos[..., np.asarray(axis)] * np.asarray(freq, dtype=np.float64))[:, None]  # [B, 1, S, n]
    if inverse:
        phi = -phi
    n = phi.shape[-1]
    a, b = (slice(0, n), slice(n, 2 * n)) if pairing == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * phi)
    out = x.copy()
    out[..., a], out[..., b] = z.real, z.imag
    return out
