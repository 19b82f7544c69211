"""The oracle's layer norm and projections against library routines, closed forms and differences."""

import numpy as np
import torch

from oracle import linear, mx, norm


def _rows(rng, *shape):
    return rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[-1])) + rng.standard_normal(shape[-1])


def test_layer_norm_against_the_library():
    rng = np.random.default_rng(1)
    x, w, b = _rows(rng, 2, 5, 24), rng.standard_normal(24), rng.standard_normal(24)
    want = torch.nn.functional.layer_norm(torch.from_numpy(x), (24,), torch.from_numpy(w), torch.from_numpy(b), 1e-5)
    assert np.allclose(norm.layer_norm(x, w, b, eps=1e-5), want.numpy(), rtol=1e-12, atol=1e-12)


def test_layer_norm_by_hand():
    # mean 2, variance 2/3 + eps 1/3 = 1: h = (-1, 0, 1)
    x = np.array([[[1.0, 2.0, 3.0]], [[4.0, 4.0, 4.0]]])
    y = norm.layer_norm(x, np.array([2.0, 3.0, 4.0]), np.ones(3), np.array([[1.0, 1.0, 0.0]] * 2), np.full((2, 3), 5.0),
                        eps=1 / 3)
    assert np.allclose(y[0, 0], [(-2 + 1) * 2 + 5, (0 + 1) * 2 + 5, 4 + 1 + 5])
    assert np.allclose(y[1, 0], [7.0, 7.0, 6.0])  # a row without variance


def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(2)
    a = [_rows(rng, 2, 3, 7), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((2, 7)),
         rng.standard_normal((2, 7))]
    dy = rng.standard_normal((2, 3, 7))
    grads = norm.layer_norm_grad(dy, *a[:4])
    for i, g in enumerate(grads):
        step = rng.standard_normal(a[i].shape)
        e = 1e-5
        f = lambda t: (norm.layer_norm(*(v + t * step if j == i else v for j, v in enumerate(a))) * dy).sum()
        # a central difference in fp64: e^2 of the third derivative and 2^-53 / e of the value
        assert abs((f(e) - f(-e)) / (2 * e) - (g * step).sum()) < 1e-6 * max(1.0, np.abs(g * step).sum())


def test_linear_rounds_its_rows_and_gradients_pass():
    rng = np.random.default_rng(3)
    w, x = rng.standard_normal((5, 64)), rng.standard_normal((2, 3, 64))
    for wf in ("mxfp4", "mxfp8"):
        codes, scales = mx.quantise(w, wf)
        packed = mx.pack(codes, wf)
        wv = mx.values(packed, scales, wf)
        for xf, most in (("mxfp4", 0.25), ("mxfp8", 2.0 ** -4)):
            xv = linear.rounded(x, xf)
            big = np.abs(x).reshape(2, 3, 2, 32).max(-1).repeat(32, -1)
            assert (np.abs(xv - x) <= most * big).all() and not np.array_equal(xv, x)
            y = linear.linear(x, packed, scales, wf, np.arange(5.0), xf)
            assert np.allclose(y, np.einsum("bsk,nk->bsn", xv, wv) + np.arange(5.0))
            assert np.allclose(linear.linear(xv, packed, scales, wf), y - np.arange(5.0))
        dy = rng.standard_normal((2, 3, 5))
        dx, db = linear.linear_grad(dy, packed, scales, wf)
        assert np.allclose(dx, np.einsum("bsn,nk->bsk", dy, wv)) and np.allclose(db, dy.sum((0, 1)))
