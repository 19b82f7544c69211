"""Projections over microscaled operands and their gradients against the fp64 oracle.

Tolerances: half a step of the result's type; K + 8 roundings of u = 2^-24 of the sum of the terms' magnitudes; with
an 8-bit side of bf16 results another 2^-10 of that sum, what the matrix instruction drops (the header states it), and, as
that is far above what normal data meet, 2^-8 of the result over all elements together (bf16 roundings are at most that,
and about a third of it in the mean)."""

import numpy as np
import pytest
import torch

from gpu_helpers import TORCH_DTYPE
from oracle import linear as oracle
from oracle import mx as oracle_mx
from paper_2609_32415_amd import ops
from paper_2609_32415_amd import _lib as L

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
PAIRS = [("mxfp4", "mxfp4"), ("mxfp8", "mxfp4"), ("mxfp4", "mxfp8"), ("mxfp8", "mxfp8")]


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _t(rng, shape, dtype, size=1.0):
    return torch.from_numpy((size * rng.standard_normal(shape)).astype(np.float32)).to("cuda:0").to(TORCH_DTYPE[dtype])


def _weights(rng, n, k, fmt):
    w = rng.standard_normal((n, k)) * np.exp(rng.standard_normal((n, 1))) / np.sqrt(k)
    codes, scales = oracle_mx.quantise(w.astype(np.float32), fmt)
    codes = oracle_mx.pack(codes, fmt)
    to = lambda a: torch.from_numpy(a).to("cuda:0")[None, None]
    return ops.MxTensor(to(codes), to(scales), fmt), (codes, scales, fmt)


def _check_y(y, xv, wv, bias, exact):
    want = xv @ wv.T
    mag = np.abs(xv) @ np.abs(wv).T
    if bias is not None:
        want = want + _np(bias)
        mag = mag + np.abs(_np(bias))
    tol = HALF[y.dtype] * np.abs(want) + (xv.shape[-1] + 8) * U * mag + (0.0 if exact else 2.0 ** -10 * mag)
    got = _np(y)
    assert got.shape == want.shape
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)
    if y.dtype == torch.bfloat16 and np.linalg.norm(want) > 0:
        assert np.linalg.norm(got - want) <= 2.0 ** -8 * np.linalg.norm(want)


def _check_linear(x, w, wp, bias, fmt, y):
    xv = oracle.rounded(_np(x), fmt)
    exact = x.dtype == torch.float32 or (fmt, wp[2]) == ("mxfp4", "mxfp4")
    _check_y(y, xv, oracle_mx.values(*wp), bias, exact)


SIZES = [(1, 1, 32, 1), (1, 1, 512, 96), (1, 3, 64, 7), (2, 5, 96, 33), (1, 17, 160, 130), (1, 33, 128, 64), (1, 61, 1536, 200),
         (3, 43, 288, 257), (1, 130, 1024, 129), (1, 257, 2080, 384), (2, 150, 544, 1153), (1, 16, 4096, 64),
         (1, 1, 4096, 1000), (1, 500, 256, 520)]


@pytest.mark.parametrize("fmt,wfmt", PAIRS)
@pytest.mark.parametrize("B,S,K,N", SIZES)
def test_product(B, S, K, N, fmt, wfmt):
    rng = np.random.default_rng(S + K + N)
    w, wp = _weights(rng, N, K, wfmt)
    for dtype in ("bf16", "f32"):
        x = _t(rng, (B, S, K), dtype, 3.0)
        bias = _t(rng, (N,), dtype) if (S + N) % 2 else None
        print("mx_linear", B, S, K, N, fmt, wfmt, dtype, flush=True)
        y = ops.mx_linear(x, w, bias, fmt=fmt)
        assert y.shape == (B, S, N) and y.dtype == x.dtype
        _check_linear(x, w, wp, bias, fmt, y)
        # the same rows as codes
        m = ops.mx_tensor((B, 1, S, K), fmt, "cuda:0")
        ops.mx_commit(x[:, None], None, m, None)
        assert torch.equal(ops.mx_linear(m, w, bias, dtype=x.dtype), y)


@pytest.mark.parametrize("wfmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,S,K,N", SIZES)
def test_gradients(B, S, K, N, dtype, wfmt):
    rng = np.random.default_rng(S + K + N)
    w, wp = _weights(rng, N, K, wfmt)
    x, bias, dy = (_t(rng, s, dtype) for s in ((B, S, K), (N,), (B, S, N)))
    x.requires_grad_()
    bias.requires_grad_()
    print("mx_linear grad", B, S, K, N, wfmt, dtype, flush=True)
    dx, db = torch.autograd.grad(ops.mx_linear(x, w, bias, fmt="mxfp8"), (x, bias), dy)
    assert dx.shape == x.shape and dx.dtype == x.dtype and db.dtype == bias.dtype
    _check_y(dx, _np(dy), oracle_mx.values(*wp).T, None, True)
    want, mag = _np(dy).sum((0, 1)), np.abs(_np(dy)).sum((0, 1))
    assert (np.abs(_np(db) - want) <= HALF[db.dtype] * np.abs(want) + (B * S + 8) * U * mag).all()


def test_fp32_gradients_keep_every_bit():
    """dy of all exponents and full significands through weights that pick one element each: dx is dy times a power of
    two, exactly, subnormals of dy's terms apart."""
    rng = np.random.default_rng(4)
    n = 96
    w = np.zeros((n, n), np.float32)
    w[rng.permutation(n), np.arange(n)] = 2.0
    codes, scales = oracle_mx.quantise(w, "mxfp4")
    m = ops.MxTensor(*(torch.from_numpy(a).to("cuda:0")[None, None] for a in (oracle_mx.pack(codes, "mxfp4"), scales)), "mxfp4")
    dy = torch.from_numpy(np.ldexp(rng.standard_normal((40, n)), rng.integers(-90, 120, (40, n))).astype(np.float32)).to("cuda:0")
    dy[0, 0] = 3.4028235e38 / 2
    dx, _ = ops.mx_linear_grad(dy, m, wanted=(True, False))
    assert np.array_equal(_np(dx), _np(dy) @ w.astype(np.float64))


def test_slices_of_rows_weights_and_results():
    rng = np.random.default_rng(5)
    K, N = 192, 320
    w, wp = _weights(rng, N, K, "mxfp4")
    wide = _t(rng, (2, 40, K + 64), "bf16")
    x = wide[:, 7:30, 32:32 + K]
    want = ops.mx_linear(x.contiguous(), w)
    assert torch.equal(ops.mx_linear(x, w), want)
    part = ops.MxTensor(w.codes[:, :, 64:256], w.scales[:, :, 64:256], "mxfp4")  # Q of a Q, K, V weight
    assert torch.equal(ops.mx_linear(x, part), want[..., 64:256])
    for pad, dt in ((1, "bf16"), (3, "f32"), (4, "bf16")):  # odd row lengths
        around = torch.full((2, 30, N + 2 * pad), 7.0, dtype=TORCH_DTYPE[dt], device="cuda:0")
        out = around[:, 3:26, pad:-pad]
        y = ops.mx_linear(x.to(TORCH_DTYPE[dt]).contiguous(), w, out=out)
        assert y is out
        assert torch.equal(y, ops.mx_linear(x.to(TORCH_DTYPE[dt]).contiguous(), w))
        out.fill_(7.0)
        assert (around == 7.0).all()
    m = ops.mx_tensor((2, 1, 30, K), "mxfp8", "cuda:0")
    ops.mx_commit(wide[:, None, :30, :K], None, m, None)
    one = m.rows(17)  # rows of each entry, not evenly spaced over the batch
    with pytest.raises(L.RefadaptError, match="evenly"):
        ops.mx_linear(one, w)
    # (sums of few rows run in another order than those of many: each against its own kind)
    first = ops.MxTensor(m.codes[:1, :, 3:20], m.scales[:1, :, 3:20], "mxfp8")
    dense = ops.MxTensor(first.codes.contiguous(), first.scales.contiguous(), "mxfp8")
    assert torch.equal(ops.mx_linear(first, w), ops.mx_linear(dense, w))
    row = ops.MxTensor(m.codes[:, :, 5:6], m.scales[:, :, 5:6], "mxfp8")  # one row of each entry
    dense = ops.MxTensor(row.codes.contiguous(), row.scales.contiguous(), "mxfp8")
    assert torch.equal(ops.mx_linear(row, w), ops.mx_linear(dense, w))
    assert torch.equal(ops.mx_linear(m, w)[:, 3:20], ops.mx_linear(m.rows(30), w)[:, 3:20])


@pytest.mark.parametrize("fmt,wfmt", PAIRS)
def test_scale_rows_at_odd_addresses(fmt, wfmt):
    """Scale rows of 5 bytes from an odd address on, the bytes around them 255 (which would make NaN of a sum)."""
    rng = np.random.default_rng(6)
    K, N, M = 160, 70, 37
    w, wp = _weights(rng, N, K, wfmt)
    x = _t(rng, (1, M, K), "bf16")
    m = ops.mx_tensor((1, 1, M, K), fmt, "cuda:0")
    ops.mx_commit(x[:, None], None, m, None)
    want = ops.mx_linear(x, w, fmt=fmt)

    def moved(t, shift, ld):
        n = t.shape[2]
        buf = torch.full((n * ld + 64,), 255, dtype=torch.uint8, device="cuda:0")
        s = buf[shift:shift + n * ld].view(1, 1, n, ld)[..., :5]
        s.copy_(t.scales)
        return ops.MxTensor(t.codes, s, t.fmt)

    for shift, ld in ((1, 5), (3, 7), (2, 6), (0, 5)):
        assert torch.equal(ops.mx_linear(moved(m, shift, ld), moved(w, shift, ld)), want), (shift, ld)


def test_non_finite_rows_and_weights():
    rng = np.random.default_rng(7)
    w, wp = _weights(rng, 96, 256, "mxfp4")
    x = _t(rng, (1, 70, 256), "bf16")
    want = ops.mx_linear(x, w, fmt="mxfp8")
    x[0, 5, 9], x[0, 64, 255] = float("nan"), float("inf")
    y = ops.mx_linear(x, w, fmt="mxfp8")
    fine = [i for i in range(70) if i not in (5, 64)]
    assert torch.isnan(y[0, [5, 64]]).all() and torch.equal(y[0, fine], want[0, fine])
    w.scales[0, 0, 33, 7] = 255
    y = ops.mx_linear(x, w, fmt="mxfp8")
    cols = [i for i in range(96) if i != 33]
    assert torch.isnan(y[..., 33]).all() and torch.equal(y[0, fine][:, cols], want[0, fine][:, cols])
    dy = _t(rng, (1, 70, 96), "bf16")
    dx, _ = ops.mx_linear_grad(dy, w)
    assert torch.isnan(dx[..., 224:]).all() and torch.isfinite(dx[..., :224]).all()


def test_largest_and_smallest_blocks():
    """Blocks at both ends of the scales: products past fp32's range are infinite, the smallest are subnormal or zero."""
    x = torch.zeros((1, 2, 64), dtype=torch.float32, device="cuda:0")
    x[0, 0, 3], x[0, 1, 40] = 2.0 ** 126, 2.0 ** -100
    w = torch.zeros((3, 64), dtype=torch.float32, device="cuda:0")
    w[0, 3], w[1, 40], w[2, 3] = 2.0 ** 100, 2.0 ** -20, 1.5
    for fmt in ("mxfp4", "mxfp8"):
        for wfmt in ("mxfp4", "mxfp8"):
            y = ops.mx_linear(x, ops.mx_weight(w, wfmt), fmt=fmt)
            assert y[0, 0, 0] == float("inf") and y[0, 0, 1] == 0 and y[0, 0, 2] == 1.5 * 2.0 ** 126
            assert y[0, 1, 0] == 0 and y[0, 1, 1] == 2.0 ** -120


def test_empty_rows():
    w, _ = _weights(np.random.default_rng(1), 48, 64, "mxfp4")
    x = torch.empty((2, 0, 64), dtype=torch.bfloat16, device="cuda:0").requires_grad_()
    b = torch.ones(48, dtype=torch.bfloat16, device="cuda:0").requires_grad_()
    y = ops.mx_linear(x, w, b)
    gx, gb = torch.autograd.grad(y, (x, b), torch.empty_like(y))
    assert y.shape == (2, 0, 48) and gx.shape == x.shape and (gb == 0).all()


def test_gradients_in_any_layout():
    rng = np.random.default_rng(8)
    for dtype, N in (("bf16", 64), ("bf16", 37), ("f32", 40)):
        w, wp = _weights(rng, N, 96, "mxfp8")
        dy = _t(rng, (2, 9, N), dtype)
        for g in (dy[:, :1, :1].expand(2, 9, N), dy.transpose(1, 2).contiguous().transpose(1, 2), dy[:1].expand(2, 9, N),
                  torch.cat((dy, dy), 1)[:, 4:13], torch.cat((dy, dy), 2)[..., 1:N + 1]):
            got = ops.mx_linear_grad(g, w)
            want = ops.mx_linear_grad(g.clone(memory_format=torch.contiguous_format), w)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_repeats_streams_and_captures():
    rng = np.random.default_rng(9)
    w, _ = _weights(rng, 384, 512, "mxfp4")
    for dtype, S in (("bf16", 200), ("f32", 33), ("bf16", 1)):
        x, b, dy = (_t(rng, s, dtype).requires_grad_(i < 2) for i, s in enumerate(((1, S, 512), (384,), (1, S, 384))))

        def step():
            y = ops.mx_linear(x, w, b, fmt="mxfp8")
            return (y.detach(), *torch.autograd.grad(y, (x, b), dy))

        want = step()
        for _ in range(3):
            assert all(torch.equal(p, q) for p, q in zip(step(), want))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        del got
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                graphs.append((g, step()))
        for rep in range(3):
            with torch.no_grad():
                x.copy_(_t(rng, x.shape, dtype))
                dy.copy_(_t(rng, dy.shape, dtype))
            torch.cuda.synchronize()
            other = torch.cuda.Stream()
            for (g, _), s in zip(graphs, (side, other)):
                with torch.cuda.stream(s):
                    g.replay()
            torch.cuda.synchronize()
            want = step()
            for _, got in graphs:
                assert all(torch.equal(p, q) for p, q in zip(got, want)), rep


def test_refusals_of_the_wrapper():
    rng = np.random.default_rng(10)
    w, _ = _weights(rng, 48, 64, "mxfp4")
    x, b = _t(rng, (2, 4, 64), "bf16"), _t(rng, (48,), "bf16")
    heads = ops.mx_tensor((1, 2, 48, 64), "mxfp4", "cuda:0")
    for call in (lambda: ops.mx_linear(x.half(), w), lambda: ops.mx_linear(x, w, b[:47]), lambda: ops.mx_linear(x, w, b.float()),
                 lambda: ops.mx_linear(x[..., :32], w), lambda: ops.mx_linear(x, w, fmt="int4"),
                 lambda: ops.mx_linear(x, heads), lambda: ops.mx_linear(heads, w), lambda: ops.mx_linear(x, w, dtype=torch.float32),
                 lambda: ops.mx_linear(x, w, out=torch.empty((2, 4, 47), dtype=x.dtype, device=x.device)),
                 lambda: ops.mx_linear(x[None], w), lambda: ops.mx_linear(x.cpu(), w), lambda: ops.mx_weight(x, "mxfp4"),
                 lambda: ops.mx_linear_grad(x, w)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(L.RefadaptError, match="workspace"):
        ops.mx_linear(_t(rng, (2, 40, 64), "bf16"), w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda:0"))
    xg, m = x.clone().requires_grad_(), ops.mx_tensor((2, 1, 4, 64), "mxfp4", "cuda:0")
    ops.mx_commit(x[:, None], None, m, None)
    with pytest.raises(ValueError, match="grad"):
        ops.mx_linear(xg, w, out=torch.empty((2, 4, 48), dtype=x.dtype, device=x.device))
    with pytest.raises(ValueError, match="grad"):
        ops.mx_linear(m, w, b.clone().requires_grad_())
    y = ops.mx_linear(xg, w)
    w.codes.add_(0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()
