"""The layer norm and its gradients against the fp64 oracle.

Tolerances count roundings, u = 2^-24 each and half a step of the result's type once. On any path of a sum there are at
most 64 additions (2 pieces of 8 elements of a lane, 6 exchanges, 16 wavefronts, and the roundings of the terms), so the
mean is off by at most 64 u mean|x|, 1 / deviation by 64 u of itself, and
h by dh = 64 u (r mean|x| + |h|)."""

import numpy as np
import pytest
import torch

from gpu_helpers import TORCH_DTYPE
from oracle import mx as oracle_mx
from oracle import norm as oracle
from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _case(seed, B, S, C, dtype, pdtype, affine, modulated, spread=1.0):
    rng = np.random.default_rng(seed)
    t = lambda a, dt: torch.from_numpy(np.asarray(a, np.float32)).to("cuda:0").to(TORCH_DTYPE[dt])
    x = t(rng.standard_normal((B, S, C)) * np.exp(0.5 * rng.standard_normal(C)) + spread * rng.standard_normal(C), dtype)
    v = lambda mean, *shape: t(mean + 0.3 * rng.standard_normal(shape), pdtype)
    p = dict(weight=v(1, C), bias=v(0, C)) if affine else dict(weight=None, bias=None)
    p.update(dict(scale=v(0, B, C), shift=v(0, B, C)) if modulated else dict(scale=None, shift=None))
    return x, p, t(rng.standard_normal((B, S, C)), dtype)


def _bounds(x, p, eps):
    """(|h|, r, dh, |w (1 + s)|, |b (1 + s)| + |t|), each [B, S, C] or broadcast to it."""
    h, r = oracle.normalised(_np(x), eps)
    C = x.shape[-1]
    m = 1.0 if p["scale"] is None else np.abs(1.0 + _np(p["scale"])[:, None])
    w = np.abs(np.ones(C) if p["weight"] is None else _np(p["weight"])) * m
    b = np.abs(np.zeros(C) if p["bias"] is None else _np(p["bias"])) * m
    t = 0.0 if p["shift"] is None else np.abs(_np(p["shift"])[:, None])
    dh = 64 * U * (r * np.abs(_np(x)).mean(-1, keepdims=True) + np.abs(h))
    return np.abs(h), r, dh, w, b + t


def _check_y(y, x, p, eps=1e-6):
    want = oracle.layer_norm(_np(x), *(_np(p[n]) for n in ("weight", "bias", "scale", "shift")), eps)
    ah, _, dh, w, b = _bounds(x, p, eps)
    tol = HALF[y.dtype] * np.abs(want) + dh * w * 1.01 + 8 * U * (ah * w + b)
    assert y.shape == x.shape and y.dtype == x.dtype
    assert (np.abs(_np(y) - want) <= tol).all(), np.max(np.abs(_np(y) - want) / tol)


def _check_grads(got, dy, x, p, eps=1e-6, chunk=64):
    want = oracle.layer_norm_grad(_np(dy), _np(x), _np(p["weight"]), _np(p["bias"]), _np(p["scale"]), eps)
    ah, r, dh, w, _ = _bounds(x, p, eps)
    g = np.abs(_np(dy))
    e = g * w
    mean = lambda a: a.mean(-1, keepdims=True)
    tol = HALF[x.dtype] * np.abs(want[0]) + 1.01 * r * (
        12 * U * e + 64 * U * mean(e) + ah * (64 * U * mean(e * ah) + mean(e * dh)) + dh * mean(e * ah)
        + 64 * U * ah * mean(e * ah))
    assert (np.abs(_np(got[0]) - want[0]) <= tol).all(), np.max(np.abs(_np(got[0]) - want[0]) / tol)
    # sums: terms within dh and 2 roundings, at most `chunk` + 4 additions in fp32
    m = 1.0 if p["scale"] is None else np.abs(1.0 + _np(p["scale"])[:, None])
    k = (chunk + 8) * U
    C = x.shape[-1]
    aw = np.abs(np.ones(C) if p["weight"] is None else _np(p["weight"]))
    ab = np.abs(np.zeros(C) if p["bias"] is None else _np(p["bias"]))
    terms = [(g * m * (dh + k * ah)).sum((0, 1)), (g * m * k).sum((0, 1)), (g * (aw * (dh + k * ah) + ab * k)).sum(1),
             (g * k).sum(1)]
    for a, b, t in zip(got[1:], want[1:], terms):
        if a is None:
            continue
        tol = HALF[a.dtype] * np.abs(b) + 1.01 * t
        assert (np.abs(_np(a).reshape(b.shape) - b) <= tol).all(), np.max(np.abs(_np(a).reshape(b.shape) - b) / tol)


SHAPES = [(1, 1, 1), (1, 3, 7), (1, 1, 1536), (2, 5, 64), (3, 33, 512), (1, 67, 520), (2, 9, 1001), (1, 130, 1024),
          (1, 12, 2048), (2, 6, 2056), (1, 5, 4096), (1, 3, 8192), (1, 2, 9000), (1, 2, 16384)]


@pytest.mark.parametrize("dtype,pdtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("B,S,C", SHAPES)
def test_forward(B, S, C, dtype, pdtype):
    for affine, modulated in ((True, True), (False, False), (S % 2 == 0, S % 2 == 1)):
        x, p, _ = _case(S + C, B, S, C, dtype, pdtype, affine, modulated)
        print("norm", B, S, C, dtype, pdtype, affine, modulated, flush=True)
        _check_y(ops.layer_norm(x, **p), x, p)


@pytest.mark.parametrize("dtype,pdtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("B,S,C", [s for s in SHAPES if s[2] <= 2056])
def test_gradients(B, S, C, dtype, pdtype):
    for affine, modulated in ((True, True), (False, False), (S % 2 == 0, S % 2 == 1)):
        x, p, dy = _case(S + C, B, S, C, dtype, pdtype, affine, modulated)
        leaves = [t.requires_grad_() for t in (x, *p.values()) if t is not None]
        print("norm grad", B, S, C, dtype, pdtype, affine, modulated, flush=True)
        y = ops.layer_norm(x, **p)
        grads = iter(torch.autograd.grad(y, leaves, dy))
        got = [next(grads) if t is not None else None for t in (x, *p.values())]
        _check_y(y.detach(), x, p)
        for t, g in zip((x, *p.values()), got):
            assert t is None or g.shape == t.shape and g.dtype == t.dtype
        _check_grads(got, dy, x, p)


def test_gradients_of_wide_rows():
    """Widths that take several pieces a lane and several wavefronts a row: dx and the sums against float64 on the GPU."""
    for S, C in ((37, 4096), (9, 8192), (5, 9000), (7, 16384)):
        x, p, dy = _case(C, 2, S, C, "f32", "f32", True, True)
        stats = torch.stack((x.mean(-1), 1 / (x.double().var(-1, correction=0) + 1e-6).sqrt().float()), -1).contiguous()
        print("norm grad wide", S, C, flush=True)
        got = ops.layer_norm_grad(dy, x, stats, p["weight"], p["bias"], scale=p["scale"])
        d = [t.double().requires_grad_() for t in (x, p["weight"], p["bias"], p["scale"], p["shift"])]
        h = (d[0] - d[0].mean(-1, keepdim=True)) / (d[0].var(-1, correction=0, keepdim=True) + 1e-6).sqrt()
        y = (h * d[1] + d[2]) * (1 + d[3][:, None]) + d[4][:, None]
        for a, b in zip(got, torch.autograd.grad(y, d, dy.double())):
            # rms: the roundings of h (64 u of a few times its size) and of the sums' terms
            assert float((a.double() - b).norm() / b.norm()) <= 64 * U


def test_columns_over_many_rows():
    """More rows than chunks hold at once: 4 rows a chunk and more, an uneven last chunk."""
    for B, S, C in ((1, 2050, 72), (3, 700, 40)):
        x, p, dy = _case(S, B, S, C, "f32", "f32", True, True)
        leaves = [t.requires_grad_() for t in (x, *p.values())]
        got = torch.autograd.grad(ops.layer_norm(x, **p), leaves, dy)
        _check_grads(got, dy, x, p)


def test_slices_and_odd_addresses():
    """Rows behind others in a larger buffer, elements at odd addresses, modulation rows of a wider tensor, a permuted
    batch; what lies around the result stays."""
    x, p, dy = _case(5, 2, 11, 96, "bf16", "bf16", True, True)
    wide = torch.randn((2, 30, 96), device="cuda:0").to(torch.bfloat16)
    wide[:, 19:] = x
    six = torch.randn((2, 6, 96), device="cuda:0").to(torch.bfloat16)
    six[:, 4], six[:, 1] = p["scale"], p["shift"]
    sliced = dict(p, scale=six[:, 4], shift=six[:, 1])
    want = ops.layer_norm(x, **p)
    assert torch.equal(ops.layer_norm(wide[:, 19:], **sliced), want)
    odd = torch.empty(2 * 11 * 97 + 1, dtype=torch.bfloat16, device="cuda:0")[1:].view(2, 11, 97)[..., :96]
    odd.copy_(x)
    assert torch.equal(ops.layer_norm(odd, **p), want)
    turned = x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(ops.layer_norm(turned, **p), want)
    around = torch.full((2, 30, 104), 7.0, dtype=torch.bfloat16, device="cuda:0")
    ops.layer_norm(x, **p, out=around[:, 3:14, 4:100])
    assert torch.equal(around[:, 3:14, 4:100], want)
    around[:, 3:14, 4:100] = 7.0
    assert (around == 7.0).all()
    ops.layer_norm(wide[:, 19:], **p, out=wide[:, 19:])
    assert torch.equal(wide[:, 19:], want)
    for y in (wide[0, 19:],):  # [S, C] rows with [C] modulation
        z = ops.layer_norm(x[0], p["weight"], p["bias"], scale=p["scale"][0], shift=p["shift"][0])
        assert torch.equal(z, y)


def test_gradients_in_any_layout_and_of_shared_modulation():
    x, p, dy = _case(6, 2, 10, 64, "f32", "f32", True, True)
    shared = p["scale"][:1].clone().requires_grad_()
    x.requires_grad_()
    y = ops.layer_norm(x, p["weight"], p["bias"], scale=shared.expand(2, 64), shift=p["shift"])
    for g in (dy[:, :1, :1].expand(2, 10, 64), dy.transpose(1, 2).contiguous().transpose(1, 2), dy[:1].expand(2, 10, 64)):
        got = torch.autograd.grad(y, (x, shared), g, retain_graph=True)
        each = dict(p, scale=shared.detach().expand(2, 64))
        want = oracle.layer_norm_grad(_np(g), _np(x), _np(p["weight"]), _np(p["bias"]), _np(each["scale"]))
        _check_grads((got[0], None, None, None, None), g, x, each)
        assert got[1].shape == (1, 64)
        assert np.allclose(_np(got[1])[0], want[3].sum(0), rtol=0, atol=1e-4)
    only = ops.layer_norm_grad(dy, x.detach(), torch.zeros((2, 10, 2), device="cuda:0") + 1, wanted=(False,) * 5)
    assert only == (None,) * 5


def test_constant_huge_and_non_finite_rows():
    x = torch.randn((1, 8, 256), device="cuda:0")
    x[0, 1] = 3.0  # no variance: h = 0
    x[0, 2] = 0.0
    x[0, 3] *= 1e15
    x[0, 4] = x[0, 4] * 1e-3 + 1e4  # a mean far above the deviation
    x[0, 5, 77] = float("nan")
    x[0, 6, 200] = float("inf")
    p = dict(weight=None, bias=None, scale=None, shift=None)
    y = ops.layer_norm(x)
    assert torch.isnan(y[0, 5]).all() and torch.isnan(y[0, 6]).all()
    assert (y[0, 1:3] == 0).all()
    fine = [0, 1, 2, 3, 4, 7]
    _check_y(y[:, fine], x[:, fine], p)
    for fmt in ("mxfp4", "mxfp8"):
        m = ops.layer_norm_mx(x, fmt)
        assert (m.scales[0, 0, 5:7] == 255).all() and (m.scales[0, 0, fine] != 255).all()
    dy = torch.randn_like(x)
    x.requires_grad_()
    gx, = torch.autograd.grad(ops.layer_norm(x), x, dy)
    assert torch.isnan(gx[0, 5:7]).all() and torch.isfinite(gx[0, fine]).all()


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,S,C", [(1, 1, 32), (2, 5, 96), (1, 17, 512), (2, 3, 1536), (1, 9, 2080), (1, 2, 8224)])
def test_codes_are_those_of_the_quantised_result(B, S, C, dtype, fmt):
    x, p, _ = _case(C, B, S, C, dtype, dtype, S % 2 == 0, True)
    y = ops.layer_norm(x, **p)
    m = ops.layer_norm_mx(x, fmt, **p)
    assert m.shape == (B, 1, S, C)
    code, scale = oracle_mx.quantise(_np(y), fmt)
    assert np.array_equal(m.scales.cpu().numpy()[:, 0], scale)
    assert np.array_equal(m.codes.cpu().numpy()[:, 0], oracle_mx.pack(code, fmt))


def test_empty_rows_and_zero_sums():
    x = torch.empty((2, 0, 64), device="cuda:0")
    assert ops.layer_norm(x).shape == (2, 0, 64)
    w, s = torch.ones(64, device="cuda:0").requires_grad_(), torch.ones((2, 64), device="cuda:0").requires_grad_()
    gw, gs = torch.autograd.grad(ops.layer_norm(x, w, scale=s), (w, s), torch.empty_like(x))
    assert (gw == 0).all() and (gs == 0).all()
    assert ops.layer_norm_mx(x, "mxfp4").shape == (2, 1, 0, 64)


def test_repeats_streams_and_captures():
    x, p, dy = _case(9, 2, 300, 768, "bf16", "f32", True, True)
    leaves = [x.requires_grad_(), *(t.requires_grad_() for t in p.values())]

    def step():
        y = ops.layer_norm(x, **p)
        return (y.detach(), *torch.autograd.grad(y, leaves, dy))

    want = step()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del got
    graphs = []
    for _ in range(2):  # two graphs with workspaces of their own, replayed at once
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            graphs.append((g, step()))
    for rep in range(3):
        with torch.no_grad():
            dy.copy_(torch.randn(dy.shape, device="cuda:0"))
            x.copy_(torch.randn(x.shape, device="cuda:0"))
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        for (g, _), s in zip(graphs, (side, other)):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = step()
        for _, got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(got, want)), rep


def test_refusals_of_the_wrapper():
    x, p, dy = _case(3, 2, 4, 64, "bf16", "bf16", True, True)
    bad = torch.zeros(64, dtype=torch.float16, device="cuda:0")
    for call in (lambda: ops.layer_norm(x.half()), lambda: ops.layer_norm(x, bad), lambda: ops.layer_norm(x, p["bias"][:63]),
                 lambda: ops.layer_norm(x, p["weight"], p["bias"].float()), lambda: ops.layer_norm(x, scale=p["scale"][:1]),
                 lambda: ops.layer_norm(x, scale=p["scale"][0]), lambda: ops.layer_norm(x[None]), lambda: ops.layer_norm(x[0, 0]),
                 lambda: ops.layer_norm(x.transpose(1, 2)), lambda: ops.layer_norm(x, out=torch.empty_like(x[:1])),
                 lambda: ops.layer_norm_mx(x, "int4"), lambda: ops.layer_norm(x.cpu()),
                 lambda: ops.layer_norm(x, p["weight"].cpu()),
                 lambda: ops.layer_norm_grad(dy, x, torch.zeros((2, 4), device="cuda:0")),
                 lambda: ops.layer_norm_grad(dy[:, :3], x, torch.zeros((2, 4, 2), device="cuda:0"))):
        with pytest.raises(ValueError):
            call()
    w = p["weight"].clone().requires_grad_()
    with pytest.raises(ValueError, match="grad"):
        ops.layer_norm(x, w, out=torch.empty_like(x))
    with pytest.raises(ValueError, match="grad"):
        ops.layer_norm_mx(x, "mxfp4", w)
    with torch.no_grad():
        ops.layer_norm(x, w, out=torch.empty_like(x))
        ops.layer_norm_mx(x, "mxfp4", w)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        xx = x.clone().requires_grad_()
        g, = torch.autograd.grad(ops.layer_norm(xx).float().square().sum(), xx, create_graph=True)
        g.float().sum().backward()
    xx = x.clone().requires_grad_()
    y = ops.layer_norm(xx * 1, w)
    with torch.no_grad():
        w.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()
