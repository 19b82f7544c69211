"""The oracle's rotary positions and block formats against closed forms and hand-derived values."""

import numpy as np
import pytest

from oracle import mx, rope


def test_rope_is_a_rotation_by_the_axis_position():
    x = np.zeros((1, 1, 3, 6))
    x[..., 0], x[..., 2], x[..., 5] = 1.0, 1.0, 7.0  # two pairs, two elements past them
    pos = np.array([[0, 0], [1, 0], [0, 2]])
    y = rope(x, pos, [np.pi / 2, np.pi / 4], [0, 1])
    assert np.allclose(y[0, 0], [[1, 0, 1, 0, 0, 7], [0, 1, 1, 0, 0, 7], [1, 0, 0, 1, 0, 7]])
    z = rope(x, pos, [np.pi / 2, np.pi / 4], [0, 1], "half")  # pairs (0, 2) and (1, 3)
    assert np.allclose(z[0, 0, 1], [-1, 0, 1, 0, 0, 7]) and np.allclose(z[0, 0, 2], [1, 0, 1, 0, 0, 7])


def test_rope_scores_depend_on_differences_and_the_inverse_undoes_it():
    r = np.random.default_rng(0)
    q, k = r.standard_normal((2, 1, 1, 5, 8))
    pos = r.integers(0, 50, (5, 2))
    freq, axis = [1.0, 0.3, 0.1, 0.01], [0, 0, 1, 1]
    f = lambda x, p: rope(x, p, freq, axis)
    assert np.allclose(f(q, pos) @ f(k, pos).swapaxes(-1, -2), f(q, pos + 11) @ f(k, pos + 11).swapaxes(-1, -2))
    assert np.allclose(rope(f(q, pos), pos, freq, axis, inverse=True), q)


def test_code_tables():
    assert mx._E4M3[-1] == 448 and mx._E4M3[1] == 2.0 ** -9 and mx._E4M3[8] == 2.0 ** -6 and len(mx._E4M3) == 127


@pytest.mark.parametrize("fmt,top,amax,byte", [
    ("mxfp4", 6.0, 6.0, 127), ("mxfp4", 6.0, 7.0, 127), ("mxfp4", 4.0, 7.0625, 128), ("mxfp4", 6.0, 3.0, 126),
    ("mxfp8", 448.0, 448.0, 127), ("mxfp8", 448.0, 464.0, 127), ("mxfp8", 240.0, 466.0, 128),
])
def test_scale_is_the_finest_that_adds_no_error(fmt, top, amax, byte):
    x = np.zeros(32)
    x[3] = -amax
    code, scale = mx.quantise(x, fmt)
    v = mx.values(mx.pack(code, fmt), scale, fmt)
    assert scale[0] == byte and v[3] == -top * 2.0 ** (byte - 127) and not v[:3].any()


def test_ties_go_to_the_even_code_and_signs_stay():
    x = np.zeros(32)
    x[:9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25]
    v = mx.values(mx.pack(mx.quantise(x, "mxfp4")[0], "mxfp4"), np.array([127]), "mxfp4")
    assert v[:9].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0] and np.signbit(v[8])


def test_ends_of_the_range():
    for fmt, lowest, highest in (("mxfp4", 0, 252), ("mxfp8", 3, 246)):
        top = 1.75 * 2.0 ** 127 if fmt == "mxfp8" else 1.5 * 2.0 ** 127
        for x, byte, want in ((0.0, lowest, 0.0), (3.3895e38, highest, top), (np.inf, 255, np.nan), (np.nan, 255, np.nan)):
            code, scale = mx.quantise(np.full(32, x), fmt)
            v = mx.values(mx.pack(code, fmt), scale, fmt)
            assert scale[0] == byte and np.array_equal(v, np.full(32, want), equal_nan=True)
    # e4m3 at the lowest scale keeps bf16's smallest values
    x = np.arange(32) * 2.0 ** -133
    assert np.array_equal(mx.values(*(lambda c, s: (mx.pack(c, "mxfp8"), s))(*mx.quantise(x, "mxfp8")), "mxfp8")[:17], x[:17])
