"""Results that share elements with the rows a call reads are refused, before anything reaches a device; slices of one
buffer that lie between each other are not (their call gets as far as the launch)."""

import random

import pytest
import torch

from paper_2609_32415_amd import _lib as L
from test_norm_linear_refusals import _linear, _linear_grad, _norm, _norm_grad, _t

HERE = 1 << 20  # an address; 2 entries of 10 rows of 256 bf16 elements below


def _overlaps(y, x, batch, rows, wy, wx):
    """By every element's address."""
    at = lambda t, w: {t.data // 2 + b * t.stride_b + s * t.stride_s + c for b in range(batch) for s in range(rows) for c in range(w)}
    return bool(at(y, wy) & at(x, wx))


BAD = [dict(ptr=HERE + 2), dict(ptr=HERE + 512), dict(ptr=HERE - 512 * 9 + 6), dict(ptr=HERE, ss=512),
       dict(ptr=HERE + 2 * 2000, sb=1 << 19), dict(ptr=HERE - 2 * (1 << 14))]


@pytest.mark.parametrize("y", BAD)
def test_parts_are_refused(y):
    x, y = _t(HERE, 1 << 14), _t(**{"sb": 1 << 14, **y})
    st, err = _norm(x=x, y=y)
    assert st == L.RA_EINVAL and "overlaps x" in err
    st, err = _norm_grad(x=x, dx=y)
    assert st == L.RA_EINVAL and "overlaps x" in err
    st, err = _norm_grad(dy=x, dx=y)
    assert st == L.RA_EINVAL and "overlaps dy" in err


@pytest.mark.parametrize("sb,ss,fits", [(512, 256, False), (255, 4096, False), (256, 512, True), (256 * 10, 256, True),
                                        (256 * 9, 256, False), (300, 512, False), (512, 1024, True)])
def test_entries_inside_each_other(sb, ss, fits):
    if fits and torch.cuda.is_available():
        pytest.skip("made-up addresses that would be launched")
    st, err = _norm(x=_t(0x100, 1 << 14), y=_t(HERE, sb, ss))
    assert ("batch entries of y overlap" in err) == (not fits), err


def test_products_are_never_in_place():
    x = _t(HERE, 40 * 256)
    for y in (x, _t(HERE + 512, 40 * 256)):
        st, err = _linear(x=x, y=y, n_out=256)
        assert st == L.RA_EINVAL and "overlaps x" in err
        st, err = _linear_grad(dy=x, dx=y, n_out=256)
        assert st == L.RA_EINVAL and "overlaps dy" in err


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses that would be launched")
def test_random_slices():
    """Both verdicts against the addresses of every element."""
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(1500):
        batch, rows, width = rng.choice((1, 2, 3)), rng.choice((1, 2, 5)), rng.choice((8, 24))
        ss = rng.choice((width, 2 * width, 3 * width + 8))
        sb = rng.choice((ss * rows, 2 * ss * rows, 3 * ss * rows + 16))
        if rng.random() < 0.2:  # entries inside each other
            sb, ss = ss, batch * ss
        kw = dict(batch=batch, rows=rows, width=width)
        x = _t(HERE, sb * rng.choice((1, 1, 1, 2)), ss)
        y = _t(HERE + 2 * rng.choice((width, ss, ss * rows, 1, 8)) * rng.randint(-4, 4), sb, ss)
        in_place = y.data == x.data and (batch == 1 or x.stride_b == sb)
        want = _overlaps(y, x, batch, rows, width, width) and not in_place
        st, err = _norm(x=x, y=y, **kw)
        assert (st == L.RA_EINVAL and "overlaps x" in err) == want, (batch, rows, width, sb, ss, y.data - HERE)
        seen[want] += 1
    assert min(seen) > 200


def test_many_entries_take_no_time():
    """65535 entries inside each other: columns of one buffer, and entries at two strides (refused)."""
    n = 65535
    x = _t(HERE, 512, n * 512)
    assert _norm(x=x, y=_t(HERE + 2, 512, n * 512), batch=n, rows=4)[0] == L.RA_EINVAL
    assert _norm(x=x, y=_t(HERE + 2, 1024, n * 512), batch=n, rows=4)[0] == L.RA_EINVAL
    if not torch.cuda.is_available():
        assert _norm(x=x, y=_t(HERE + 512, 512, n * 512), batch=n, rows=4)[0] not in (L.RA_OK, L.RA_EINVAL)  # to the launch
