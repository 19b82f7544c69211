"""Rotary positions against the fp64 oracle, their refusals of wrong tensors, and graph replays.

Tolerance: one rounding to the run dtype (at most eps / 2 of the value) plus the fp32 arithmetic of a pair of length
r: the angle within an eighth of a turn (3 roundings of at most pi/4), cos and sin (2 each) and the two products and
their sum (3), below 8 roundings of 2^-24 r; the angle's reduction adds 2^-52 |phi| r.
"""

import numpy as np
import pytest
import torch

from gpu_helpers import TORCH_DTYPE
from oracle import rope as oracle_rope
from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu

AXES = {64: (8, 28, 28), 128: (16, 56, 56), 96: (32, 32)}


def _tensor(rng, B, H, S, D, dtype, layout="bhsd"):
    x = torch.from_numpy(rng.standard_normal((B, H, S, D)).astype(np.float32)).to(TORCH_DTYPE[dtype]).to("cuda:0")
    if layout == "bshd":
        return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    if layout == "padded":  # rows of a wider, longer buffer
        buf = torch.zeros((B, H, S + 3, D + 16), dtype=x.dtype, device="cuda:0")
        buf[:, :, :S, 8:8 + D] = x
        return buf[:, :, :S, 8:8 + D]
    return x


def _check(y, x, pos, freq, axis, pairing, inverse, dtype):
    xs = x.double().cpu().numpy()
    p = pos.double().cpu().numpy()
    want = oracle_rope(xs, p, freq.numpy(), axis.numpy(), pairing, inverse)
    got = y.double().cpu().numpy()
    n = freq.numel()
    r = np.zeros_like(xs)
    a, b = (slice(0, n), slice(n, 2 * n)) if pairing == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    r[..., a] = r[..., b] = np.hypot(xs[..., a], xs[..., b])
    phi = np.abs(p).max() * float(freq.abs().max()) if p.size else 0.0
    half = torch.finfo(TORCH_DTYPE[dtype]).eps / 2
    tol = half * np.abs(want) * (1 + 2 * half) + r * (2.0 ** -21 + 2.0 ** -52 * phi) + 2.0 ** -133
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())
    assert np.array_equal(got[..., 2 * n:], xs[..., 2 * n:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", ["interleaved", "half"])
@pytest.mark.parametrize("B,H,S,D,layout", [(1, 1, 1, 64, "bhsd"), (2, 3, 77, 64, "bshd"), (1, 24, 129, 128, "bhsd"),
                                            (2, 5, 33, 96, "padded"), (3, 2, 257, 128, "padded"), (1, 70, 2, 128, "bshd")])
def test_rope_matches_the_oracle(dtype, pairing, B, H, S, D, layout):
    rng = np.random.default_rng(B + 10 * H + S + D)
    freq, axis = ops.rope_frequencies(AXES[D])
    q, k = (_tensor(rng, B, H, S, D, dtype, layout) for _ in range(2))
    pos = torch.from_numpy(rng.integers(-40, 4096, (B, S, len(AXES[D]))).astype(np.int32)).to("cuda:0")
    q0, k0 = q.clone(), k.clone()
    print("rope", dtype, pairing, B, H, S, D, layout, flush=True)
    yq, yk = ops.rope(q, k, pos=pos, freq=freq, axis=axis, pairing=pairing)
    back = ops.rope(yq, pos=pos, freq=freq, axis=axis, pairing=pairing, inverse=True)
    torch.cuda.synchronize()
    _check(yq, q, pos, freq, axis, pairing, False, dtype)
    _check(yk, k, pos, freq, axis, pairing, False, dtype)
    _check(back, yq, pos, freq, axis, pairing, True, dtype)
    assert torch.equal(q, q0) and torch.equal(k, k0)
    # in place: the same bits
    ops.rope(q, k, pos=pos, freq=freq, axis=axis, pairing=pairing, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(q, yq) and torch.equal(k, yk)


@pytest.mark.parametrize("pos_dtype", [torch.int32, torch.float32])
@pytest.mark.parametrize("n", [1, 3, 8, 13, 31])
def test_pairs_that_end_inside_a_piece_and_shared_or_far_positions(pos_dtype, n):
    """Any number of interleaved pairs; elements past them keep their bits, infinities and NaN among them;
    positions shared by the batch, of a view with a stride, up to 2^24 (and fractions of it as fp32)."""
    rng = np.random.default_rng(n)
    B, H, S, D = 2, 3, 41, 64
    x = _tensor(rng, B, H, S, D, "f32")
    wide = torch.from_numpy(rng.integers(0, 1 << 24, (S, 5)).astype(np.float64))
    if pos_dtype == torch.float32:
        wide = wide / 8
    pos = wide.to(pos_dtype).to("cuda:0")[:, :2]
    freq = torch.from_numpy(np.concatenate([[1.0], rng.uniform(0, 2, n - 1)]))
    axis = torch.from_numpy((np.arange(n) % 2).astype(np.int32))
    y = ops.rope(x, pos=pos, freq=freq, axis=axis)
    torch.cuda.synchronize()
    _check(y, x, pos, freq, axis, "interleaved", False, "f32")
    x[..., 2 * n:] = torch.tensor([float("inf"), float("nan")], device="cuda:0").repeat(D // 2 - n)
    y = ops.rope(x, pos=pos, freq=freq, axis=axis)
    torch.cuda.synchronize()
    assert torch.equal(y[..., 2 * n:].view(torch.int32), x[..., 2 * n:].view(torch.int32))
    assert torch.isfinite(y[..., :2 * n]).all()


def test_nothing_is_written_outside_the_rows():
    B, H, S, D = 1, 2, 9, 64
    buf = torch.full((B, H, S + 2, D), 3.0, dtype=torch.bfloat16, device="cuda:0")
    freq, axis = ops.rope_frequencies((32, 32))
    pos = torch.arange(2 * S, dtype=torch.int32, device="cuda:0").view(S, 2)
    x = torch.randn((B, H, S, D), device="cuda:0").to(torch.bfloat16)
    ops.rope(x, pos=pos, freq=freq, axis=axis, q_out=buf[:, :, 1:S + 1])
    torch.cuda.synchronize()
    assert (buf[:, :, 0] == 3).all() and (buf[:, :, S + 1] == 3).all()
    e = ops.rope(x[:, :, :0], pos=pos[:0], freq=freq, axis=axis)  # no rows: nothing to do
    assert e.shape == (B, H, 0, D)


def test_infinite_position_gives_nan_and_leaves_other_rows_alone():
    x = torch.ones((1, 1, 3, 64), device="cuda:0")
    freq, axis = ops.rope_frequencies((64,))
    y = ops.rope(x, pos=torch.tensor([[1.0], [float("inf")], [2.0]], device="cuda:0"), freq=freq, axis=axis)
    torch.cuda.synchronize()
    assert torch.isnan(y[0, 0, 1]).all() and torch.isfinite(y[0, 0, [0, 2]]).all()


def test_gradient_is_the_inverse_turn():
    """<inverse(dy), h> against the difference quotient of <dy, rope(x + t h)>, fp32 data, sums in fp64."""
    rng = np.random.default_rng(5)
    freq, axis = ops.rope_frequencies((16, 24, 24))
    pos = torch.from_numpy(rng.integers(0, 200, (2, 19, 3)).astype(np.int32)).to("cuda:0")
    x, h, dy = (_tensor(rng, 2, 3, 19, 64, "f32") for _ in range(3))
    f = lambda t: ops.rope(t, pos=pos, freq=freq, axis=axis).double()
    dx = ops.rope(dy, pos=pos, freq=freq, axis=axis, inverse=True)
    diff = ((f(x + 0.5 * h) - f(x - 0.5 * h)) * dy.double()).sum()
    # the map is linear: the quotient is exact but for roundings, a few 2^-24 of each of the terms
    scale = (x.double().abs() + h.double().abs()).mul(dy.double().abs()).sum()
    assert abs(float((dx.double() * h.double()).sum() - diff)) <= 32 * 2.0 ** -24 * float(scale) * 2


def test_graph_replays_follow_new_positions():
    freq, axis = ops.rope_frequencies((16, 24, 24))
    q = torch.zeros((1, 4, 65, 64), dtype=torch.bfloat16, device="cuda:0")
    pos = torch.zeros((65, 3), dtype=torch.int32, device="cuda:0")
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        ops.rope(q, pos=pos, freq=freq, axis=axis, q_out=out)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            ops.rope(q, pos=pos, freq=freq, axis=axis, q_out=out)
    for rep in range(3):
        q.copy_(torch.randn(q.shape, device="cuda:0"))
        pos.copy_(torch.randint(0, 999, pos.shape, device="cuda:0"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ops.rope(q, pos=pos, freq=freq, axis=axis))


def test_wrong_tensors_are_refused():
    x = torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16, device="cuda:0")
    pos = torch.zeros((5, 1), dtype=torch.int32, device="cuda:0")
    freq, axis = ops.rope_frequencies((64,))
    ok = dict(pos=pos, freq=freq, axis=axis)
    for bad in (dict(ok, pos=pos.long()), dict(ok, pos=pos[:4]), dict(ok, pos=pos.cpu()), dict(ok, freq=freq.float()),
                dict(ok, freq=freq.to("cuda:0")), dict(ok, axis=axis[:3]), dict(ok, pairing="pairs"),
                dict(ok, pos=pos.expand(3, 5, 1)), dict(ok, k_out=x), dict(ok, q_out=x.cpu()),
                dict(ok, q_out=x[:, :, :4])):
        with pytest.raises(ValueError):
            ops.rope(x, **bad)
    with pytest.raises(ValueError):
        ops.rope(x.half(), **ok)
    with pytest.raises(ValueError):
        ops.rope(x, x[:, :1], **ok)
    torch.cuda.synchronize()
