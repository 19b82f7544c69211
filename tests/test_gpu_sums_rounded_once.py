"""Sums of gradients that leave fp64 for bf16 are rounded once: sums next to the middle of two bf16 values, nearer to it
than fp32 tells."""

import math

import numpy as np
import pytest
import torch

from paper_2609_32415_amd import ops
from test_gpu_mx_linear import _weights

pytestmark = pytest.mark.gpu

# (a, b, c): a + b is halfway between two bf16 values, c is on one side of it
MIDDLES = [(s * 2.0 ** e * a, s * 2.0 ** (e - 8), s * 2.0 ** (e - 30) * c)
           for s in (1, -1) for e in (0, 5, -60, 100) for a in (1.0, 1.0 + 2.0 ** -7) for c in (1, -1)]


def _once(v):
    """The bf16 value nearest to v, which is far from the ends of the range; the even one of two."""
    step = 2.0 ** (math.frexp(v)[1] - 8)
    return round(v / step) * step  # exact: powers of two, and Python's round of halves is to even


def _dy(rows, behind):
    """Rows of which the first two add up to the middles, and row ``behind``, of another chunk, holds the rest."""
    dy = torch.zeros((rows, len(MIDDLES)), dtype=torch.float64)
    for i, (a, b, c) in enumerate(MIDDLES):
        dy[0, i], dy[1, i], dy[behind, i] = a, b, c
    bits = dy.to(torch.bfloat16)
    assert torch.equal(bits.double(), dy)
    return bits.to("cuda:0"), [_once(a + b + c) for a, b, c in MIDDLES]


def test_expected():
    assert _once(1.0 + 2.0 ** -8 + 2.0 ** -30) == 1.0 + 2.0 ** -7 and _once(1.0 + 2.0 ** -8) == 1.0
    twice = [_once(float(np.float32(a + b + c))) for a, b, c in MIDDLES]
    assert sum(_once(a + b + c) != t for (a, b, c), t in zip(MIDDLES, twice)) == len(MIDDLES) // 2


def test_norm():
    dy, want = _dy(4, 2)  # two chunks of two rows
    C = dy.shape[1]
    x = torch.ones((4, C), dtype=torch.bfloat16, device="cuda:0")
    stats = torch.tensor([0.0, 1.0], device="cuda:0").expand(4, 2).contiguous()  # h = x = 1
    got = ops.layer_norm_grad(dy, x, stats, wanted=(False, True, True, True, True))[1:]
    for t in got:
        assert t.dtype == torch.bfloat16 and t.flatten().tolist() == want
    # two entries: dweight and dbias are twice that
    got = ops.layer_norm_grad(dy.expand(2, 4, C), x.expand(2, 4, C), stats.expand(2, 4, 2).contiguous(),
                              wanted=(False, True, True, True, True))[1:]
    for t, f in zip(got, (2, 2, 1, 1)):
        assert all(row == [f * v for v in want] for row in t.view(-1, C).tolist())


def test_projection():
    dy, want = _dy(48, 20)  # three chunks of 16 rows
    w, _ = _weights(np.random.default_rng(0), dy.shape[1], 32, "mxfp4")
    _, db = ops.mx_linear_grad(dy, w, wanted=(False, True))
    assert db.tolist() == want


def test_not_finite():
    """Sums past the largest bf16 and fp32 values, infinities and NaN."""
    inf = math.inf
    top = float(torch.finfo(torch.bfloat16).max)
    cols = [(top, top, 0.0), (-top, -top, 0.0), (inf, 1.0, 1.0), (inf, 0.0, -inf), (math.nan, 0.0, 1.0),
            (0.0, 0.0, 0.0), (top, 0.0, top * 2.0 ** -30)]
    dy = torch.zeros((48, len(cols)), dtype=torch.bfloat16)
    for i, (a, b, c) in enumerate(cols):
        dy[0, i], dy[1, i], dy[20, i] = a, b, c
    w, _ = _weights(np.random.default_rng(0), len(cols), 32, "mxfp4")
    _, db = ops.mx_linear_grad(dy.to("cuda:0"), w, wanted=(False, True))
    want = torch.tensor([inf, -inf, inf, math.nan, math.nan, 0.0, top], dtype=torch.bfloat16)
    assert torch.equal(db.cpu().nan_to_num(nan=-7.0), want.nan_to_num(nan=-7.0))
