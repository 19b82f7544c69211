"""The ends of fp32's range, as the header states them: rows of the layer norm whose sum, or the sum of whose squares,
passes it, and gradients of projections too small for three bf16 terms."""

import pytest
import torch

from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [64, 1001, 4096])
def test_norm(C):
    x = torch.randn((1, 4, C), generator=torch.Generator().manual_seed(0)).to("cuda:0")
    x[0, 1] *= 2.0 ** 70  # squares
    x[0, 2] = 3e38  # the sum
    weight, bias = torch.full((C,), 2.0, device="cuda:0"), torch.arange(C, device="cuda:0").float()
    y = ops.layer_norm(x, weight, bias)
    assert torch.equal(y[0, 1], bias) and y[0, 2].isnan().all()
    assert torch.equal(y[:, ::3], ops.layer_norm(x[:, ::3].contiguous(), weight, bias))


def _gradient(dy):
    """dy [8] times a weight of 2^100, by the gradient's product."""
    w = torch.zeros((32, 32), device="cuda:0")
    w[:8, :8] = torch.eye(8, device="cuda:0") * 2.0 ** 100
    rows = torch.zeros((1, 32), device="cuda:0")
    rows[0, :8] = dy
    return ops.mx_linear_grad(rows, ops.mx_weight(w, "mxfp4"))[0][0, :8].double() * 2.0 ** -100


@pytest.mark.parametrize("e", [-149, -140, -134, -133, -126, -118, -111, -110, -109, -50, 0, 20])
def test_small_gradients(e):
    step = max(2.0 ** (e - 23), 2.0 ** -149)
    odd = torch.tensor([0, 1, 3, 0x155555, 0x2aaaab, 0x7fffff, 0x400001, 0x7f0001], dtype=torch.float64)
    dy = torch.clamp(2.0 ** e + torch.minimum(odd, torch.tensor(2.0 ** e / step - 1)) * step, max=2.0 ** (e + 1) - step)
    assert torch.equal(dy.float().double(), dy)
    dy = dy.to("cuda:0")
    got = _gradient(dy.float())
    if e >= -110:
        assert torch.equal(got, dy)
    else:
        assert ((dy - got >= 0) & (dy - got < 2.0 ** -133)).all()
    assert torch.equal(_gradient(-dy.float()), -got)
