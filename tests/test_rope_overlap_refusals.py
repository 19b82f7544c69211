"""refadapt_rope refuses outputs that overlap what the launch still reads or writes (no GPU needed)."""

import pytest

from paper_2609_32415_amd import _lib as L
from test_rope_mx_refusals import _rope, _t


@pytest.mark.parametrize("kw,msg", [
    # a broadcast input in place: every head (batch entry) would turn the same rows once more
    (dict(q=_t(0x9000, sb=1280, sh=0), qo=_t(0x9000, sb=1280, sh=0)), "q is broadcast"),
    (dict(batch=2, heads=1, q=_t(0x9000), qo=_t(0x9000)), "q is broadcast"),
    (dict(batch=2, q=_t(0x9000, sb=2560, sh=1280), qo=_t(0x9000, sb=2560, sh=1280), k=_t(0x20000, sh=1280),
          ko=_t(0x20000, sh=1280)), "k is broadcast"),
    # one buffer twice: both outputs, or an output that the other tensor is read from
    (dict(q=_t(0x1000, sh=1280), k=_t(0x1000, sh=1280), qo=_t(0x9000, sh=1280), ko=_t(0x9000, sh=1280)), "overlap"),
    (dict(q=_t(0x1000, sh=1280), k=_t(0x9000, sh=1280), qo=_t(0x9000, sh=1280), ko=_t(0x20000, sh=1280)), "overlap"),
    (dict(q=_t(0x1000, sh=1280), k=_t(0x9000, sh=1280), qo=_t(0x20000, sh=1280), ko=_t(0x1000, sh=1280)), "overlap"),
    (dict(q=_t(0x1000, sh=1280), k=_t(0x1000, sh=1280), qo=_t(0x1000, sh=1280), ko=_t(0x1000, sh=1280)), "overlap"),
])
def test_overlap(kw, msg):
    st, err = _rope(**kw)
    assert st == L.RA_EINVAL and msg in err, (st, err)
