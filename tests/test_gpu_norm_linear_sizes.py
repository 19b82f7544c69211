"""Layer norms and projections at the sizes where their kernels change: every tile, the border between few rows and tiles,
many batch entries, and tensors whose offsets pass 32 bits. Tolerances as beside the kernels' other tests."""

import numpy as np
import pytest
import torch

from oracle import mx as oracle_mx
from paper_2609_32415_amd import ops
from test_gpu_mx_linear import HALF, PAIRS, U, _check_linear, _check_y, _np, _t, _weights
from test_gpu_norm import _case, _check_grads, _check_y as _check_norm

pytestmark = pytest.mark.gpu


# tiles of 64 in four stages and (more than one a CU) in two, of 128 (more than three of 64 a CU) and of 256; rows and outputs that end inside a tile; K of one stage, of an
# odd and an even number, and ending inside one
TILES = [(1, 63, 32, 65), (2, 65, 416, 127), (1, 1100, 352, 1101), (3, 400, 1056, 1200), (1, 1801, 160, 1795), (3, 601, 288, 1800), (1, 2300, 96, 3839), (2, 1153, 352, 3848)]


@pytest.mark.parametrize("fmt,wfmt", PAIRS)
@pytest.mark.parametrize("B,S,K,N", TILES)
def test_tiles(B, S, K, N, fmt, wfmt):
    rng = np.random.default_rng(S + K + N)
    w, wp = _weights(rng, N, K, wfmt)
    for dtype in ("bf16", "f32"):
        x, bias = _t(rng, (B, S, K), dtype, 3.0), _t(rng, (N,), dtype)
        around = torch.full((B, S + 3, N + 9), 7.0, dtype=x.dtype, device="cuda:0")
        out = around[:, 2:-1, 8:-1]  # whole 16-byte units where N + 9 is
        print("tiles", B, S, K, N, fmt, wfmt, dtype, flush=True)
        y = ops.mx_linear(x, w, bias, fmt=fmt, out=out)
        _check_linear(x, w, wp, bias, fmt, y)
        assert torch.equal(ops.mx_linear(x, w, bias, fmt=fmt), y)
        out.fill_(7.0)
        assert (around == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,K,N", [(1801, 1824, 33), (2300, 3840, 136), (1153, 96, 1795), (1100, 1120, 264)])
def test_gradient_tiles(S, K, N, dtype):
    rng = np.random.default_rng(S + K + N)
    w, wp = _weights(rng, N, K, "mxfp4")
    dy = _t(rng, (1, S, N), dtype)
    print("gradient tiles", S, K, N, dtype, flush=True)
    dx, db = ops.mx_linear_grad(dy, w)
    _check_y(dx, _np(dy), oracle_mx.values(*wp).T, None, True)
    want, mag = _np(dy).sum((0, 1)), np.abs(_np(dy)).sum((0, 1))
    assert (np.abs(_np(db) - want) <= HALF[db.dtype] * np.abs(want) + (S + 8) * U * mag).all()


@pytest.mark.parametrize("fmt,wfmt", PAIRS)
@pytest.mark.parametrize("B,S,K,N", [(2, 16, 1536, 96), (1, 32, 160, 70), (32, 1, 96, 40), (1, 31, 2080, 33), (1, 33, 160, 70),
                                     (1, 2, 32768, 40), (1, 1, 131072, 33), (3, 4, 1536, 9001)])
def test_few_rows(B, S, K, N, fmt, wfmt):
    """Up to 32 rows; rows that fill the place in LDS, and that do not fit in it."""
    rng = np.random.default_rng(S + K + N)
    w, wp = _weights(rng, N, K, wfmt)
    for dtype in ("bf16", "f32"):
        x, bias = _t(rng, (B, S, K), dtype, 3.0), _t(rng, (N,), dtype)
        print("few rows", B, S, K, N, fmt, wfmt, dtype, flush=True)
        y = ops.mx_linear(x, w, bias, fmt=fmt)
        _check_linear(x, w, wp, bias, fmt, y)
        m = ops.mx_tensor((B, 1, S, K), fmt, "cuda:0")
        ops.mx_commit(x[:, None], None, m, None)
        assert torch.equal(ops.mx_linear(m, w, bias, dtype=x.dtype), y)


@pytest.mark.parametrize("B,S,C", [(300, 3, 72), (700, 1, 40), (5, 120, 9000)])
def test_norm_gradients_of_many_entries(B, S, C):
    """More batch entries than chunks of rows."""
    x, p, dy = _case(B, B, S, C, "f32", "f32", True, True)
    leaves = [t.requires_grad_() for t in (x, *p.values())]
    got = torch.autograd.grad(ops.layer_norm(x, **p), leaves, dy)
    if C <= 2056:
        _check_grads(got, dy, x, p, chunk=B)
    d = [t.detach().double().requires_grad_() for t in leaves]
    h = (d[0] - d[0].mean(-1, keepdim=True)) / (d[0].var(-1, correction=0, keepdim=True) + 1e-6).sqrt()
    y = (h * d[1] + d[2]) * (1 + d[3][:, None]) + d[4][:, None]
    for a, b in zip(got, torch.autograd.grad(y, d, dy.double())):
        assert float((a.double() - b).norm() / b.norm()) <= 64 * U


def test_norm_of_very_many_rows():
    x, p, dy = _case(1, 1, 70001, 24, "bf16", "f32", True, True)
    _check_norm(ops.layer_norm(x, **p), x, p)


FAR = 1 << 28  # elements from one row to the next: offsets of 10 rows pass 2^31 elements


def test_offsets_past_32_bits():
    """Rows of x, dy, y and codes in buffers of more than 2^32 bytes, against the same rows close together."""
    buf = torch.zeros(10 * FAR, dtype=torch.bfloat16, device="cuda:0")
    far = buf.as_strided((1, 10, 192), (0, FAR, 1))
    x, p, dy = _case(2, 1, 10, 192, "bf16", "bf16", True, True)
    far.copy_(x)
    want = ops.layer_norm(x, **p)
    assert torch.equal(ops.layer_norm(far, **p), want)
    leaf = x.clone().requires_grad_()
    near, = torch.autograd.grad(ops.layer_norm(leaf, **p), leaf, dy)
    leaf = far.detach().requires_grad_()
    got, = torch.autograd.grad(ops.layer_norm(leaf, **p), leaf, dy)
    assert torch.equal(got, near)
    per_entry = buf.as_strided((10, 1, 192), (FAR, 192, 1))  # entries far apart
    many = dict(p, scale=p["scale"].expand(10, 192), shift=p["shift"].expand(10, 192))
    assert torch.equal(ops.layer_norm(per_entry, **many)[:, 0], want[0])
    w, _ = _weights(np.random.default_rng(3), 192, 192, "mxfp4")
    assert torch.equal(ops.mx_linear(far, w), ops.mx_linear(x, w))
    _, db = ops.mx_linear_grad(far, w, wanted=(False, True))
    assert torch.equal(db, ops.mx_linear_grad(x, w, wanted=(False, True))[1])
    want = ops.mx_linear(x, w)
    assert torch.equal(ops.mx_linear(x, w, out=far), want)
    ops.layer_norm(x, **p, out=far)
    assert torch.equal(far, ops.layer_norm(x, **p))
    code = buf.view(torch.uint8)
    for fmt, n in (("mxfp4", 96), ("mxfp8", 192)):
        m = ops.mx_tensor((1, 1, 10, 192), fmt, "cuda:0")
        spread = ops.MxTensor(code.as_strided((1, 1, 10, n), (0, 0, 2 * FAR, 1)), m.scales.clone(), fmt)
        ops.layer_norm_mx(x, fmt, **p, out=m)
        ops.layer_norm_mx(x, fmt, **p, out=spread)
        assert torch.equal(spread.codes, m.codes) and torch.equal(spread.scales, m.scales)
    del buf, far, per_entry, code, spread, leaf, got


def test_products_past_32_bits():
    """40 rows far apart in y (tiles), and 70000 rows of 32768 elements, whose codes take more than 2^31 bytes."""
    rng = np.random.default_rng(4)
    w, wp = _weights(rng, 72, 96, "mxfp8")
    x = _t(rng, (1, 40, 96), "bf16")
    buf = torch.zeros(40 * FAR // 2, dtype=torch.bfloat16, device="cuda:0")
    out = buf.as_strided((1, 40, 72), (0, FAR // 2, 1))
    assert torch.equal(ops.mx_linear(x, w, out=out), ops.mx_linear(x, w))
    far = buf.as_strided((1, 40, 96), (0, FAR // 2, 1))
    far.copy_(x)
    assert torch.equal(ops.mx_linear(far, w), ops.mx_linear(x, w))
    dy = _t(rng, (1, 40, 72), "bf16")
    want = ops.mx_linear_grad(dy, w)
    out.copy_(dy)
    got = ops.mx_linear_grad(out, w)  # rows too far apart for the product are copied
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del buf, out, far
    M, K, N = 70000, 32768, 40
    w, wp = _weights(rng, N, K, "mxfp4")
    x = torch.randn((1, M, K), dtype=torch.bfloat16, device="cuda:0")
    y = ops.mx_linear(x, w, fmt="mxfp8")
    rows = [0, 1, 65535, 65536, M - 130, M - 1]
    _check_linear(x[:, rows], w, wp, None, "mxfp8", y[:, rows])
    for r0 in (0, 50000, M - 2000):  # the same sums in a call of their own
        assert torch.equal(ops.mx_linear(x[:, r0:r0 + 2000].contiguous(), w, fmt="mxfp8"), y[:, r0:r0 + 2000])


def test_two_calls_at_once():
    """Calls on two streams that overlap, each with a workspace of its own."""
    rng = np.random.default_rng(5)
    w, _ = _weights(rng, 1536, 1024, "mxfp4")
    xs = [_t(rng, (1, 900, 1024), "bf16") for _ in range(2)]
    want = [ops.mx_linear(x, w, fmt="mxfp8") for x in xs]
    n = [ops.layer_norm(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((ops.mx_linear(xs[i], w, fmt="mxfp8"), ops.layer_norm(xs[i])))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, want[i]) and torch.equal(b, n[i]) for a, b in got[i])


@pytest.mark.parametrize("dtype,pdtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("C", [9, 511, 513, 1023, 1999, 3001, 5003, 9001, 16383])
def test_norm_of_odd_widths(C, dtype, pdtype):
    """Rows at every alignment that end inside a lane's piece; what lies between and around them stays."""
    x, p, dy = _case(C, 2, 5, C, dtype, pdtype, True, True)
    for pad in (1, 2):
        around = torch.full((2, 7, C + pad), 7.0, dtype=x.dtype, device="cuda:0")
        out = around[:, 1:-1, :-pad]
        print("odd width", C, dtype, pdtype, pad, flush=True)
        with torch.no_grad():
            _check_norm(ops.layer_norm(x, **p, out=out), x, p)
        out.fill_(7.0)
        assert (around == 7.0).all()
    leaves = [t.requires_grad_() for t in (x, *p.values())]
    got = torch.autograd.grad(ops.layer_norm(x, **p), leaves, dy)
    d = [t.detach().double().requires_grad_() for t in leaves]
    h = (d[0] - d[0].mean(-1, keepdim=True)) / (d[0].var(-1, correction=0, keepdim=True) + 1e-6).sqrt()
    y = (h * d[1] + d[2]) * (1 + d[3][:, None]) + d[4][:, None]
    for a, b in zip(got, torch.autograd.grad(y, d, dy.double())):
        # rms: the roundings of h (64 u of a few times its size), of the sums' terms and of the result
        assert float((a.double() - b).norm() / b.norm()) <= 64 * U + HALF[a.dtype]


def test_codes_of_rows_at_odd_addresses():
    for dtype, pad in (("bf16", 1), ("f32", 3)):
        x, p, _ = _case(8, 2, 5, 2080, dtype, dtype, True, True)
        odd = torch.empty((2, 5, 2080 + pad), dtype=x.dtype, device="cuda:0")[..., pad:]
        odd.copy_(x)
        for fmt in ("mxfp4", "mxfp8"):
            a, b = ops.layer_norm_mx(odd, fmt, **p), ops.layer_norm_mx(x, fmt, **p)
            assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)


def test_slices_of_one_buffer():
    """Rows, columns and entries of one buffer that lie between each other's, as rows and as results."""
    x, p, dy = _case(11, 2, 6, 128, "bf16", "bf16", True, True)
    want, w = ops.layer_norm(x, **p), _weights(np.random.default_rng(1), 128, 128, "mxfp4")[0]
    product = ops.mx_linear(x, w)
    shapes = [lambda b: (b[..., :128], b[..., 128:256]), lambda b: (b[:, :6, :128], b[:, 6:, :128]),
              lambda b: (b[:, ::2, :128], b[:, 1::2, :128]), lambda b: (b[:, 1::2, 128:256], b[:, ::2, :128])]
    for cut in shapes:
        for call, result in ((lambda i, o: ops.layer_norm(i, **p, out=o), want), (lambda i, o: ops.mx_linear(i, w, out=o), product)):
            buf = torch.zeros((2, 12, 256), dtype=torch.bfloat16, device="cuda:0")
            src, dst = cut(buf)
            src, dst = src[:, :6], dst[:, :6]
            src.copy_(x)
            call(src, dst)
            assert torch.equal(dst, result) and torch.equal(src, x)
    with pytest.raises(RuntimeError, match="overlaps"):
        ops.layer_norm(x[:, :5], **p, out=x[:, 1:])
    with pytest.raises(RuntimeError, match="overlaps"):
        ops.mx_linear(x, w, out=x)
