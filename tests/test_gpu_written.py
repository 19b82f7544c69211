"""The wrappers' writes into tensors that a recorded call saved are refused by its backward pass; writes elsewhere, also
while a graph is captured, change nothing."""

import pytest
import torch

from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu


def _x(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.bfloat16).to("cuda:0")


def test_a_norm_in_place_of_saved_rows():
    x, w, dy = _x(0, 2, 9, 64), _x(1, 64).requires_grad_(), _x(2, 2, 9, 64)
    y = ops.layer_norm(x, w)
    want, = torch.autograd.grad(y, w, dy, retain_graph=True)
    with torch.no_grad():
        ops.layer_norm(x, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y, w, dy)
    x = _x(0, 2, 9, 64)
    y = ops.layer_norm(x, w)
    ops.layer_norm(x, out=torch.empty_like(x))
    assert torch.equal(torch.autograd.grad(y, w, dy)[0], want)


def test_weights_quantised_again():
    x, w = _x(3, 1, 40, 64).requires_grad_(), ops.mx_weight(_x(4, 48, 64), "mxfp4")
    y = ops.mx_linear(x, w)
    ops.mx_commit(_x(5, 1, 1, 48, 64), None, w, None)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(torch.ones_like(y))


def test_captured_and_in_inference_mode():
    x, w = _x(6, 1, 40, 64), ops.mx_weight(_x(7, 48, 64), "mxfp4")
    want = ops.mx_linear(ops.layer_norm(x), w)
    n, y = torch.empty_like(x), torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.mx_linear(ops.layer_norm(x, out=n), w, out=y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    with torch.inference_mode():
        y = torch.empty_like(want)
        assert torch.equal(ops.mx_linear(ops.layer_norm(x, out=torch.empty_like(x)), w, out=y), want)
