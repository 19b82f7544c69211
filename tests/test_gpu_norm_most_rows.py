"""The layer norm and its gradients at the largest number of rows: 2^31 - 1, each written once, none behind them."""

import pytest
import torch

from paper_2609_32415_amd import ops
from test_gpu_mx_linear import HALF, U

pytestmark = pytest.mark.gpu

S, N = (1 << 31) - 1, 64  # rows repeat with this period


def _filled(pattern):
    t = torch.empty((S + 1, 2), dtype=torch.bfloat16, device="cuda:0")
    t.view(-1, N, 2).copy_(pattern.expand(1 << 25, N, 2))
    return t


def _check(t, want, untouched=None):
    """``t`` [S, 2 or the like] repeats ``want``; the row behind the last is ``untouched``."""
    whole = t[:S // N * N].view(-1, N, 2)
    for a in range(0, len(whole), 1 << 22):
        assert (whole[a:a + (1 << 22)] == want).all()
    assert (t[S // N * N:S] == want[:S % N]).all()
    if untouched is not None:
        assert (t[S:] == untouched).all()


def test_every_row():
    g = torch.Generator().manual_seed(0)
    cases = [torch.randn((N, 2), generator=g).to(torch.bfloat16).to("cuda:0") for _ in range(2)]
    weight, bias = torch.tensor([1.5, -0.5], device="cuda:0"), torch.tensor([0.25, 3.0], device="cuda:0")
    with torch.no_grad():
        want = ops.layer_norm(cases[0][None], weight, bias)[0]
    x = _filled(cases[0])
    print("rows", S, flush=True)
    y = torch.full_like(x, 7.0)
    with torch.no_grad():
        ops.layer_norm(x[None, :S], weight, bias, out=y[None, :S])
    _check(y, want, 7.0)
    del y
    leaves = [t.requires_grad_() for t in (cases[0].clone()[None], weight.clone(), bias.clone())]
    few = torch.autograd.grad(ops.layer_norm(*leaves), leaves, cases[1][None])
    dy = _filled(cases[1])
    leaves = [t.requires_grad_() for t in (x[None, :S], weight, bias)]
    print("gradients of rows", S, flush=True)
    dx, dw, db = torch.autograd.grad(ops.layer_norm(*leaves), leaves, dy[None, :S])
    _check(dx[0], few[0][0])
    # The sums are of 2^25 periods less the last row, each of N terms. fp32 within a chunk of rows: off by a rounding a
    # row at most, of the sum of the terms' sizes. (Terms h g are a few roundings off: 16 of them.)
    with torch.no_grad():
        d = cases[0].double() - cases[0].double().mean(-1, keepdim=True)
        h = d / (d.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    for got, terms in ((dw, cases[1].double() * h), (db, cases[1].double())):
        exact = terms.sum(0) * (1 << 25) - terms[N - 1]
        size = terms.abs().sum(0) * (1 << 25)
        longest = -(-S // 512) / 4  # rows of a chunk that a wavefront adds up
        assert ((got.double() - exact).abs() <= (longest + 16) * U * size + HALF[torch.float32] * exact.abs()).all()
