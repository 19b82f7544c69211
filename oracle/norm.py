"""Layer norm of hidden rows with an affine map and a block's modulation, and its gradients, in fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

The gradients come from the norm's Jacobian, row by row: with h = (x - mean) / s and s = sqrt(var + eps),
dh_i / dx_j = (delta_ij - 1/C - h_i h_j / C) / s.
"""

from __future__ import annotations

import numpy as np


def layer_norm(x, weight=None, bias=None, scale=None, shift=None, eps=1e-6):
    """``x`` [B, S, C], ``weight`` and ``bias`` [C], ``scale`` and ``shift`` [B, C]."""
    h = normalised(x, eps)[0]
    n = h * (1.0 if weight is None else np.asarray(weight, np.float64)) + (
        0.0 if bias is None else np.asarray(bias, np.float64))
    m = 0.0 if scale is None else np.asarray(scale, np.float64)[:, None]
    t = 0.0 if shift is None else np.asarray(shift, np.float64)[:, None]
    return n * (1.0 + m) + t


def normalised(x, eps):
    """(h, 1 / s) of rows."""
    x = np.asarray(x, dtype=np.float64)
    d = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return d * r, r


def layer_norm_grad(dy, x, weight=None, bias=None, scale=None, eps=1e-6):
    """The gradients (dx, dweight, dbias, dscale, dshift)."""
    dy = np.asarray(dy, dtype=np.float64)
    h, r = normalised(x, eps)
    B, S, C = h.shape
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(C) if bias is None else np.asarray(bias, np.float64)
    m = np.zeros((B, C)) if scale is None else np.asarray(scale, np.float64)
    dx = np.empty_like(h)
    eye = np.eye(C)
    for i in range(B):
        e = dy[i] * (1.0 + m[i]) * w
        for s in range(S):
            jac = (eye - 1.0 / C - np.outer(h[i, s], h[i, s]) / C) * r[i, s]
            dx[i, s] = e[s] @ jac
    n = h * w + b
    return (dx, (dy * (1.0 + m[:, None]) * h).sum((0, 1)), (dy * (1.0 + m[:, None])).sum((0, 1)), (dy * n).sum(1),
            dy.sum(1))
