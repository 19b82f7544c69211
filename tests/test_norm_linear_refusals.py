"""refadapt_layer_norm, refadapt_mx_linear and their gradients reject malformed arguments before anything reaches a
device (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2609_32415_amd import _lib as L
from paper_2609_32415_amd import ops

NONE, NO_MX = L.ra_tensor(0, 0, 0, 0), L.ra_mx_tensor(0, 0, 0, 0, 0, 0, 0, 0)
BIG = 1 << 40


def _t(ptr=0x1000, sb=1 << 20, ss=256):
    return L.ra_tensor(ptr, sb, 0, ss)


def _m(codes=0x1000, sb=1 << 20, ss=128, scales=0x2000, eb=1 << 16, es=8):
    return L.ra_mx_tensor(codes, sb, 0, ss, scales, eb, 0, es)


def _call(name, desc, args):
    return getattr(L.LIB, "refadapt_" + name)(ctypes.byref(desc), ctypes.byref(args), None), L.refadapt_last_error()


def _norm(x=_t(), y=_t(0x9000), y_mx=NO_MX, weight=None, bias=None, scale=None, shift=None, scale_stride=0,
          shift_stride=0, stats=None, **kw):
    d = dict(batch=2, rows=10, width=256, dtype=L.RA_BF16, param_dtype=L.RA_BF16, format=L.RA_MXFP4, eps=1e-6)
    d.update(kw)
    return _call("layer_norm", L.ra_norm_desc(**d),
                 L.ra_norm_args(x, y, y_mx, weight, bias, scale, shift, scale_stride, shift_stride, stats))


SIZES = [
    (dict(batch=0), L.RA_EINVAL, "sizes"),
    (dict(rows=-1), L.RA_EINVAL, "sizes"),
    (dict(width=0), L.RA_EINVAL, "sizes"),
    (dict(dtype=2), L.RA_EINVAL, "dtype"),
    (dict(dtype=L.RA_F32), L.RA_EINVAL, "parameters"),
    (dict(param_dtype=5), L.RA_EINVAL, "parameters"),
    (dict(eps=-1.0), L.RA_EINVAL, "eps"),
    (dict(eps=float("nan")), L.RA_EINVAL, "eps"),
    (dict(width=16385), L.RA_EUNSUPPORTED, "width"),
    (dict(batch=65536), L.RA_EUNSUPPORTED, "too many"),
    (dict(batch=64, rows=1 << 25), L.RA_EUNSUPPORTED, "too many"),
]


@pytest.mark.parametrize("kw,status,msg", SIZES + [
    (dict(x=NONE), L.RA_EINVAL, "null x"),
    (dict(y=NONE), L.RA_EINVAL, "null y"),
    (dict(x=_t(ss=255)), L.RA_EINVAL, "row stride"),
    (dict(x=_t(sb=-1)), L.RA_EINVAL, "negative"),
    (dict(x=_t(0x1001)), L.RA_EUNSUPPORTED, "aligned"),
    (dict(y=_t(0x9000, sb=255)), L.RA_EINVAL, "overlap"),
    (dict(x=_t(0x9000, sb=0)), L.RA_EINVAL, "in place"),
    (dict(weight=0x1001), L.RA_EUNSUPPORTED, "weight"),
    (dict(shift=0x1001), L.RA_EUNSUPPORTED, "shift"),
    (dict(scale=0x1000, scale_stride=-2), L.RA_EINVAL, "negative"),
    (dict(stats=0x1004), L.RA_EUNSUPPORTED, "stats"),
    (dict(y_mx=_m()), L.RA_EINVAL, "both"),
    (dict(y=NONE, y_mx=_m(), format=2), L.RA_EINVAL, "format"),
    (dict(y=NONE, y_mx=_m(), width=250), L.RA_EUNSUPPORTED, "multiple of 32"),
    (dict(y=NONE, y_mx=_m(scales=0)), L.RA_EINVAL, "null"),
    (dict(y=NONE, y_mx=_m(codes=0x1008)), L.RA_EUNSUPPORTED, "16-byte"),
    (dict(y=NONE, y_mx=_m(es=10)), L.RA_EUNSUPPORTED, "scales"),
    (dict(y=NONE, y_mx=_m(ss=64)), L.RA_EINVAL, "row strides"),
    (dict(y=NONE, y_mx=_m(sb=0)), L.RA_EINVAL, "overlap"),
])
def test_layer_norm(kw, status, msg):
    st, err = _norm(**kw)
    assert st == status and msg in err, (st, err)


def _norm_grad(dy=_t(), x=_t(0x5000), dx=_t(0x9000), stats=0x8000, weight=None, bias=None, scale=None, scale_stride=0,
               dweight=0x3000, dbias=None, dscale=None, dshift=None, workspace=0x10000, nbytes=BIG, **kw):
    d = dict(batch=2, rows=10, width=256, dtype=L.RA_BF16, param_dtype=L.RA_BF16, format=0, eps=1e-6)
    d.update(kw)
    return _call("layer_norm_grad", L.ra_norm_desc(**d),
                 L.ra_norm_grad_args(dy, x, dx, stats, weight, bias, scale, scale_stride, dweight, dbias, dscale, dshift,
                                     workspace, nbytes))


@pytest.mark.parametrize("kw,status,msg", SIZES + [
    (dict(dy=NONE), L.RA_EINVAL, "null dy"),
    (dict(x=NONE), L.RA_EINVAL, "null x"),
    (dict(stats=None), L.RA_EINVAL, "stats"),
    (dict(stats=0x8004), L.RA_EUNSUPPORTED, "stats"),
    (dict(dx=NONE, dweight=None), L.RA_EINVAL, "no gradient"),
    (dict(dx=_t(0x9000, sb=0)), L.RA_EINVAL, "overlap"),
    (dict(dx=_t(0x9000, ss=128)), L.RA_EINVAL, "row stride"),
    (dict(dx=_t(0x1000), dy=_t(0x1000, sb=0)), L.RA_EINVAL, "broadcast"),
    (dict(dweight=0x3001), L.RA_EUNSUPPORTED, "dweight"),
    (dict(scale_stride=-1), L.RA_EINVAL, "negative"),
    (dict(workspace=None), L.RA_EWORKSPACE, "workspace"),
    (dict(nbytes=100), L.RA_EWORKSPACE, "workspace"),
    (dict(workspace=0x10008), L.RA_EUNSUPPORTED, "16-byte"),
])
def test_layer_norm_grad(kw, status, msg):
    st, err = _norm_grad(**kw)
    assert st == status and msg in err, (st, err)


def _linear(x=_t(), x_mx=NO_MX, w=_m(0x4000), bias=None, y=_t(0x9000), workspace=0x10000, nbytes=BIG, **kw):
    d = dict(batch=2, rows=40, n_in=256, n_out=100, dtype=L.RA_BF16, x_format=L.RA_MXFP8, w_format=L.RA_MXFP4)
    d.update(kw)
    return _call("mx_linear", L.ra_linear_desc(**d), L.ra_linear_args(x, x_mx, w, bias, y, workspace, nbytes))


LINEAR_SIZES = [
    (dict(batch=0), L.RA_EINVAL, "sizes"),
    (dict(rows=-1), L.RA_EINVAL, "sizes"),
    (dict(n_out=0), L.RA_EINVAL, "sizes"),
    (dict(dtype=3), L.RA_EINVAL, "dtype"),
    (dict(x_format=2), L.RA_EINVAL, "formats"),
    (dict(w_format=-1), L.RA_EINVAL, "formats"),
    (dict(n_in=100), L.RA_EUNSUPPORTED, "multiple of 32"),
    (dict(n_in=1 << 22), L.RA_EUNSUPPORTED, "above"),
    (dict(n_out=1 << 22), L.RA_EUNSUPPORTED, "above"),
    (dict(batch=65536), L.RA_EUNSUPPORTED, "too many"),
    (dict(batch=1, rows=1 << 24), L.RA_EUNSUPPORTED, "too many"),
    (dict(w=NO_MX), L.RA_EINVAL, "w: null"),
    (dict(w=_m(0x4008)), L.RA_EUNSUPPORTED, "16-byte"),
    (dict(w=_m(ss=64)), L.RA_EINVAL, "row strides"),
    (dict(w=_m(es=9)), L.RA_EUNSUPPORTED, "scales"),
    (dict(w=_m(ss=(1 << 22) + 16)), L.RA_EUNSUPPORTED, "row stride of w"),
    (dict(workspace=None), L.RA_EWORKSPACE, "workspace"),
    (dict(nbytes=1000), L.RA_EWORKSPACE, "workspace"),
    (dict(workspace=0x10004), L.RA_EUNSUPPORTED, "16-byte"),
]


@pytest.mark.parametrize("kw,status,msg", LINEAR_SIZES + [
    (dict(x=NONE), L.RA_EINVAL, "null"),
    (dict(x_mx=_m(ss=256)), L.RA_EINVAL, "both"),
    (dict(x=_t(0x1008)), L.RA_EUNSUPPORTED, "16-byte"),
    (dict(x=_t(ss=260)), L.RA_EUNSUPPORTED, "multiples"),
    (dict(x=_t(ss=128)), L.RA_EINVAL, "row stride"),
    (dict(x=NONE, x_mx=_m(ss=256, sb=10240, es=8, eb=328)), L.RA_EUNSUPPORTED, "evenly"),
    (dict(x=NONE, x_mx=_m(ss=256, sb=12288, es=8, eb=320)), L.RA_EUNSUPPORTED, "evenly"),
    (dict(x=NONE, x_mx=_m(ss=128)), L.RA_EINVAL, "row strides"),
    (dict(x=NONE, batch=1, x_mx=_m(ss=1 << 23)), L.RA_EUNSUPPORTED, "row stride of x_mx"),
    (dict(y=NONE), L.RA_EINVAL, "null y"),
    (dict(y=_t(0x9001)), L.RA_EUNSUPPORTED, "aligned"),
    (dict(y=_t(0x9000, ss=99)), L.RA_EINVAL, "row stride"),
    (dict(y=_t(0x9000, sb=99)), L.RA_EINVAL, "overlap"),
    (dict(bias=0x3001), L.RA_EUNSUPPORTED, "bias"),
])
def test_mx_linear(kw, status, msg):
    st, err = _linear(**kw)
    assert st == status and msg in err, (st, err)


def _linear_grad(dy=_t(), w=_m(0x4000), dx=_t(0x9000), dbias=0x3000, workspace=0x10000, nbytes=BIG, **kw):
    d = dict(batch=2, rows=40, n_in=256, n_out=104, dtype=L.RA_BF16, x_format=L.RA_MXFP8, w_format=L.RA_MXFP4)
    d.update(kw)
    return _call("mx_linear_grad", L.ra_linear_desc(**d), L.ra_linear_grad_args(dy, w, dx, dbias, workspace, nbytes))


@pytest.mark.parametrize("kw,status,msg", LINEAR_SIZES + [
    (dict(dx=NONE, dbias=None), L.RA_EINVAL, "no gradient"),
    (dict(dy=NONE), L.RA_EINVAL, "null dy"),
    (dict(dy=_t(0x1002)), L.RA_EUNSUPPORTED, "evenly"),
    (dict(dy=_t(sb=10248)), L.RA_EUNSUPPORTED, "evenly"),
    (dict(dy=_t(ss=1 << 22), batch=1), L.RA_EUNSUPPORTED, "row stride of dy"),
    (dict(dx=_t(0x9001)), L.RA_EUNSUPPORTED, "aligned"),
    (dict(dx=_t(0x9000, ss=255)), L.RA_EINVAL, "row stride"),
    (dict(dx=_t(0x9000, sb=0), dy=_t(sb=10240)), L.RA_EINVAL, "overlap"),
    (dict(dbias=0x3001, dy=_t(sb=10240)), L.RA_EUNSUPPORTED, "dbias"),
])
def test_mx_linear_grad(kw, status, msg):
    kw = dict(kw)
    if "dy" not in kw:
        kw["dy"] = _t(sb=10240)
    st, err = _linear_grad(**kw)
    assert st == status and msg in err, (st, err)


def test_null_blocks_and_nothing_to_do():
    for name in ("layer_norm", "layer_norm_grad", "mx_linear", "mx_linear_grad"):
        assert getattr(L.LIB, "refadapt_" + name)(None, None, None) == L.RA_EINVAL
    assert _norm(rows=0, x=NONE, y=NONE)[0] == L.RA_OK
    assert _norm_grad(rows=0, dy=NONE, x=NONE, dx=_t(), dweight=None, stats=None)[0] == L.RA_OK
    assert _linear(rows=0, x=NONE, y=NONE)[0] == L.RA_OK
    assert _linear_grad(rows=0, dy=NONE, dbias=None)[0] == L.RA_OK


def test_workspace_sizes():
    d = L.ra_linear_desc(2, 40, 256, 104, L.RA_BF16, L.RA_MXFP8, L.RA_MXFP4)
    size = L.LIB.refadapt_mx_linear_workspace_size
    assert size(d, 0) >= 80 * (256 + 8) and size(d, 1) == 0
    f = L.ra_linear_desc(2, 40, 256, 104, L.RA_F32, L.RA_MXFP8, L.RA_MXFP4)
    assert size(f, 1) >= (80 + 104) * 512 and size(f, 0) > size(f, 1)
    few = L.ra_linear_desc(2, 10, 256, 104, L.RA_BF16, L.RA_MXFP8, L.RA_MXFP4)
    assert size(few, 0) == 0  # rounded on the way
    assert L.LIB.refadapt_mx_linear_grad_workspace_size(d) >= 256 * 104 * 2 + 104 * 4
    assert L.LIB.refadapt_mx_linear_grad_workspace_size(f) >= 256 * 104 * 2 + 3 * 80 * 104 * 2
    bad = L.ra_linear_desc(2, 40, 250, 104, L.RA_BF16, L.RA_MXFP8, L.RA_MXFP4)
    assert size(bad, 0) == 0 and L.LIB.refadapt_mx_linear_grad_workspace_size(bad) == 0
    n = L.ra_norm_desc(3, 100, 512, L.RA_BF16, L.RA_F32, 0, 1e-6)
    assert L.LIB.refadapt_layer_norm_grad_workspace_size(n) >= 3 * 2 * 512 * 4
    n.width = 20000
    assert L.LIB.refadapt_layer_norm_grad_workspace_size(n) == 0


def test_wrappers_refuse_host_tensors():
    x, w = torch.zeros((2, 4, 64)), torch.zeros((48, 64))
    m = ops.MxTensor(torch.zeros((1, 1, 48, 32), dtype=torch.uint8), torch.zeros((1, 1, 48, 2), dtype=torch.uint8), "mxfp4")
    if torch.cuda.is_available():
        pytest.skip("the device tests cover these")
    for call in (lambda: ops.layer_norm(x), lambda: ops.layer_norm(x.requires_grad_()), lambda: ops.layer_norm_mx(x.detach(), "mxfp4"),
                 lambda: ops.layer_norm_grad(x, x, torch.zeros((2, 4, 2))), lambda: ops.mx_weight(w, "mxfp4"),
                 lambda: ops.mx_linear(x.detach(), m), lambda: ops.mx_linear_grad(torch.zeros((2, 4, 48)), m)):
        with pytest.raises((ValueError, RuntimeError)):
            call()
