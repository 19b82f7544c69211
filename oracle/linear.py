"""Projections over microscaled operands and their gradients, in fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""

from __future__ import annotations

import numpy as np

from . import mx


def rounded(x, fmt):
    """The values that rows stand for after their rounding to ``fmt``."""
    codes, scales = mx.quantise(x, fmt)
    return mx.values(mx.pack(codes, fmt), scales, fmt)


def linear(x, w_codes, w_scales, w_fmt, bias=None, fmt=None):
    """Rows [..., K] rounded to ``fmt`` (None: as they are) times the weights' values [N, K], plus ``bias`` [N]."""
    x = np.asarray(x, dtype=np.float64) if fmt is None else rounded(x, fmt)
    y = x @ mx.values(w_codes, w_scales, w_fmt).T
    return y if bias is None else y + np.asarray(bias, np.float64)


def linear_grad(dy, w_codes, w_scales, w_fmt):
    """(dx, dbias) of ``dy`` [..., N]: the rounding of the rows passes gradients on as they are."""
    dy = np.asarray(dy, dtype=np.float64)
    return dy @ mx.values(w_codes, w_scales, w_fmt), dy.reshape(-1, dy.shape[-1]).sum(0)
