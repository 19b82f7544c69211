"""Gradients through ``ops.rope``: those of its inputs are the turn back of those of its outputs.

The turn back of fp32 data is the same kernel on the same numbers, so it is compared for equality; against the fp64
formula the tolerance is test_gpu_rope's (8 roundings of 2^-24 of a pair's length, and one of the output).
"""

import numpy as np
import pytest
import torch

from gpu_helpers import TORCH_DTYPE
from oracle import rope as oracle_rope
from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu

B, H, S, D = 2, 3, 37, 64


def _case(dtype, pairing="interleaved", seed=0):
    rng = np.random.default_rng(seed)
    t = lambda: torch.from_numpy(rng.standard_normal((B, H, S, D)).astype(np.float32)).to(TORCH_DTYPE[dtype]).to("cuda:0")
    freq, axis = ops.rope_frequencies((16, 16, 16))  # the last 16 elements are copied
    pos = torch.from_numpy(rng.integers(0, 500, (B, S, 3)).astype(np.int32)).to("cuda:0")
    return t, dict(pos=pos, freq=freq, axis=axis, pairing=pairing)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["interleaved", "half"])
@pytest.mark.parametrize("inverse", [False, True])
def test_both_gradients(dtype, pairing, inverse):
    t, kw = _case(dtype, pairing)
    q, k, dq, dk = t().requires_grad_(), t().requires_grad_(), t(), t()
    yq, yk = ops.rope(q, k, inverse=inverse, **kw)
    assert yq.requires_grad and yk.requires_grad
    with torch.no_grad():
        plain = ops.rope(q, k, inverse=inverse, **kw)
    assert not plain[0].requires_grad and torch.equal(yq, plain[0]) and torch.equal(yk, plain[1])
    torch.autograd.backward((yq, yk), (dq, dk))
    want = ops.rope(dq, dk, inverse=not inverse, **kw)
    torch.cuda.synchronize()
    assert torch.equal(q.grad, want[0]) and torch.equal(k.grad, want[1])
    xs = dq.double().cpu().numpy()
    exact = oracle_rope(xs, kw["pos"].cpu().numpy(), kw["freq"].numpy(), kw["axis"].numpy(), pairing, not inverse)
    half = torch.finfo(TORCH_DTYPE[dtype]).eps / 2
    n = kw["freq"].numel()
    r = np.zeros_like(xs)
    a, b = (slice(0, n), slice(n, 2 * n)) if pairing == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    r[..., a] = r[..., b] = np.hypot(xs[..., a], xs[..., b])
    assert (np.abs(q.grad.double().cpu().numpy() - exact) <= half * np.abs(exact) * (1 + 2 * half) + 2.0 ** -21 * r).all()


def test_one_of_two_inputs_and_one_of_two_outputs():
    t, kw = _case("f32")
    dq = t()
    q, k = t().requires_grad_(), t()
    yq, yk = ops.rope(q, k, **kw)
    assert yq.requires_grad and not yk.requires_grad
    yq.backward(dq)
    q2, k2 = t().requires_grad_(), t().requires_grad_()
    ops.rope(q2, k2, **kw)[1].backward(dq)  # q2's output is not used
    want = ops.rope(dq, inverse=True, **kw)
    torch.cuda.synchronize()
    assert torch.equal(q.grad, want) and k.grad is None and torch.equal(k2.grad, want) and q2.grad is None


def test_against_differences_and_twice():
    """Through a nonlinear loss: the directional derivative in fp32, and the second derivative (the map is linear, so
    that of sum(y^4) / 4 along h is 3 <y^2, rope(h)^2>)."""
    t, kw = _case("f32")
    x, h = t().requires_grad_(), t()
    y = ops.rope(x, **kw)
    g, = torch.autograd.grad((y ** 4).sum() / 4, x, create_graph=True)
    second, = torch.autograd.grad((g * h).sum(), x)
    with torch.no_grad():
        want = 3 * (y.double() ** 2 * ops.rope(h, **kw).double() ** 2).sum()
        got = (second.double() * h.double()).sum()
        # every term of the sum is a product of a few fp32 results, each within 8 roundings of 2^-24 of its pair's length
        pair = lambda z: z.double().view(*z.shape[:-1], -1, 2).norm(dim=-1)
        assert abs(float(got - want)) <= 64 * 2.0 ** -24 * float((3 * pair(y) ** 2 * pair(h) ** 2).sum()) * 2
        e = 2.0 ** -7
        f = lambda s: (ops.rope(x + s * h, **kw).double() ** 4).sum() / 4
        slope = (f(e) - f(-e)) / (2 * e)
        # the central difference of a quartic is off by e^2 times its cubic coefficient, sum(y rope(h)^3); roundings of
        # the two sums are divided by 2 e
        cubic = (y.double() * ops.rope(h, **kw).double() ** 3).abs().sum()
        tol = e * e * float(cubic) + 64 * 2.0 ** -24 * float((pair(y) + e * pair(h)).pow(4).sum()) / e
        assert abs(float((g.double() * h.double()).sum() - slope)) <= tol


def test_gradients_of_other_layouts():
    """A gradient with stride 0 (of a sum), one whose head dimension is not contiguous, and one at an odd address."""
    t, kw = _case("bf16")
    ones = torch.ones((B, H, S, D), dtype=torch.bfloat16, device="cuda:0")
    spread = torch.randn((B, H, D, S), device="cuda:0").to(torch.bfloat16).transpose(2, 3)
    odd = torch.randn(B * H * S * D + 1, device="cuda:0").to(torch.bfloat16)[1:].view(B, H, S, D)
    for dy in (ones[:1, :1, :1, :1].expand(B, H, S, D), spread, odd):
        q = t().requires_grad_()
        ops.rope(q, **kw).backward(dy)
        want = ops.rope(dy.clone(memory_format=torch.contiguous_format), inverse=True, **kw)
        torch.cuda.synchronize()
        assert torch.equal(q.grad, want)
    heads = t().permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # heads beside the channels
    q = heads.clone().requires_grad_()
    (ops.rope(q, **kw).float() ** 2).sum().backward()
    torch.cuda.synchronize()
    assert torch.isfinite(q.grad).all()


def test_tables_changed_before_the_backward_are_noticed():
    t, kw = _case("f32")
    q = t().requires_grad_()
    y = ops.rope(q, **kw)
    kw["pos"].add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_outputs_in_place_and_gradients_of_the_tables_are_refused():
    t, kw = _case("f32")
    q, k, buf = t().requires_grad_(), t(), t()
    for call in (lambda: ops.rope(q, q_out=buf, **kw), lambda: ops.rope(q, q_out=q, **kw),
                 lambda: ops.rope(k, q, k_out=buf, **kw), lambda: ops.rope(k, q_out=q, **kw),
                 lambda: ops.rope(k, **{**kw, "pos": kw["pos"].float().requires_grad_()}),
                 lambda: ops.rope(k, **{**kw, "freq": kw["freq"].clone().requires_grad_()})):
        with pytest.raises(ValueError, match="grad"):
            call()
    with torch.no_grad():  # nothing is recorded: as ever
        want = ops.rope(q, **kw)
        ops.rope(q, q_out=buf, **kw)
        ops.rope(q, q_out=q, **kw)
    torch.cuda.synchronize()
    assert torch.equal(buf, want) and torch.equal(q, want)


def test_backward_on_another_stream_and_captured():
    t, kw = _case("f32")
    dy = t()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q = t().requires_grad_()
    with torch.cuda.stream(s):
        out = ops.rope(q, **kw)
        g0, = torch.autograd.grad(out, q, dy)
    torch.cuda.synchronize()
    assert torch.equal(g0, ops.rope(dy, inverse=True, **kw))
    del out, g0  # the eager graph is gone before the capture
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            gq, = torch.autograd.grad(ops.rope(q, **kw), q, dy)
    for rep in range(3):
        dy.copy_(torch.randn(dy.shape, device="cuda:0"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(gq, ops.rope(dy, inverse=True, **kw)), rep
