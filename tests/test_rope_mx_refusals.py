"""refadapt_rope, refadapt_mx_commit, refadapt_mx_read and refadapt_joint_attn_mx reject malformed arguments before
anything reaches a device (no GPU needed)."""

import ctypes

import pytest

from paper_2609_32415_amd import _lib as L


def _t(ptr=0x1000, sb=0, sh=0, ss=128):
    return L.ra_tensor(ptr, sb, sh, ss)


def _m(codes=0x1000, ss=64, scales=0x2000, es=4, sh=0, eh=0):
    return L.ra_mx_tensor(codes, 0, sh, ss, scales, 0, eh, es)


NONE, NO_MX = L.ra_tensor(0, 0, 0, 0), L.ra_mx_tensor(0, 0, 0, 0, 0, 0, 0, 0)


def _rope(freq=(1.0, 0.5), axis=(0, 1), q=_t(), k=NONE, qo=_t(0x9000), ko=NONE, pos=0x1000, tables=True, **kw):
    f, a = (ctypes.c_double * len(freq))(*freq), (ctypes.c_int32 * len(axis))(*axis)
    d = dict(batch=1, heads=2, rows=10, head_dim=128, dtype=L.RA_BF16, n_pairs=len(freq), pairing=L.RA_ROPE_INTERLEAVED,
             n_axes=2, inverse=0, pos_dtype=L.RA_POS_I32, pos_stride_b=0, pos_stride_s=2,
             freq=ctypes.addressof(f) if tables else None, axis=ctypes.addressof(a))
    d.update(kw)
    st = L.LIB.refadapt_rope(ctypes.byref(L.ra_rope_desc(**d)), ctypes.byref(L.ra_rope_args(q, k, qo, ko, pos)), None)
    return st, L.refadapt_last_error()


@pytest.mark.parametrize("kw,status,msg", [
    (dict(batch=0), L.RA_EINVAL, "sizes"),
    (dict(rows=-1), L.RA_EINVAL, "sizes"),
    (dict(dtype=2), L.RA_EINVAL, "dtype"),
    (dict(pos_dtype=2), L.RA_EINVAL, "pos_dtype"),
    (dict(pairing=2), L.RA_EINVAL, "pairing"),
    (dict(head_dim=100), L.RA_EUNSUPPORTED, "head_dim"),
    (dict(n_pairs=0), L.RA_EINVAL, "n_pairs"),
    (dict(n_pairs=65), L.RA_EINVAL, "n_pairs"),
    (dict(n_pairs=129, head_dim=512), L.RA_EUNSUPPORTED, "n_pairs"),
    (dict(pairing=L.RA_ROPE_HALF), L.RA_EUNSUPPORTED, "multiples of 8"),
    (dict(n_axes=0), L.RA_EINVAL, "n_axes"),
    (dict(n_axes=9), L.RA_EINVAL, "n_axes"),
    (dict(axis=(0, 2)), L.RA_EINVAL, "axis[1]"),
    (dict(axis=(-1, 0)), L.RA_EINVAL, "axis[0]"),
    (dict(freq=(float("nan"), 1.0)), L.RA_EINVAL, "freq[0]"),
    (dict(tables=False), L.RA_EINVAL, "freq"),
    (dict(pos_stride_s=-1), L.RA_EINVAL, "position stride"),
    (dict(pos=None), L.RA_EINVAL, "pos"),
    (dict(pos=0x1002), L.RA_EUNSUPPORTED, "pos"),
    (dict(q=_t(0)), L.RA_EINVAL, "q:"),
    (dict(qo=_t(0x9008)), L.RA_EUNSUPPORTED, "q_out"),
    (dict(k=_t()), L.RA_EINVAL, "k_out"),
    (dict(ko=_t()), L.RA_EINVAL, "k:"),
    (dict(q=_t(ss=64)), L.RA_EINVAL, "row stride"),
    (dict(batch=1 << 20, rows=1 << 10), L.RA_EUNSUPPORTED, "too large"),
])
def test_rope(kw, status, msg):
    st, err = _rope(**kw)
    assert st == status and msg in err, (st, err)


def test_rope_of_no_rows_and_null_desc():
    assert _rope(rows=0, q=NONE, qo=NONE, pos=None)[0] == L.RA_OK
    assert L.LIB.refadapt_rope(None, ctypes.byref(L.ra_rope_args()), None) == L.RA_EINVAL
    assert L.LIB.refadapt_rope(ctypes.byref(L.ra_rope_desc()), None, None) == L.RA_EINVAL


CASES = [
    (dict(batch=0), L.RA_EINVAL, "sizes"),
    (dict(n_ref=-1), L.RA_EINVAL, "sizes"),
    (dict(dtype=3), L.RA_EINVAL, "dtype"),
    (dict(fmt=2), L.RA_EINVAL, "format"),
    (dict(head_dim=48), L.RA_EUNSUPPORTED, "head_dim"),
    (dict(heads=65536), L.RA_EUNSUPPORTED, "65535"),
    (dict(n_ref=(1 << 27) + 1), L.RA_EUNSUPPORTED, "too many"),
    (dict(k=_t(0)), L.RA_EINVAL, "k_"),
    (dict(km=NO_MX), L.RA_EINVAL, "k_mx"),
    (dict(km=_m(scales=0)), L.RA_EINVAL, "k_mx"),
    (dict(v=_t()), L.RA_EINVAL, "v_mx"),
    (dict(vm=_m()), L.RA_EINVAL, "v_"),
    (dict(q=_t()), L.RA_EINVAL, "q_mx"),
    (dict(km=_m(codes=0x1008)), L.RA_EUNSUPPORTED, "16-byte"),
    (dict(km=_m(ss=72)), L.RA_EUNSUPPORTED, "16-byte"),
    (dict(km=_m(ss=48)), L.RA_EINVAL, "row strides"),
    (dict(km=_m(es=2)), L.RA_EINVAL, "row strides"),
    (dict(km=_m(es=6)), L.RA_EUNSUPPORTED, "scales"),
    (dict(km=_m(scales=0x2002)), L.RA_EUNSUPPORTED, "scales"),
    (dict(km=_m(eh=-4)), L.RA_EINVAL, "negative"),
]


def _call(fn, batch=1, heads=2, n_ref=10, head_dim=128, dtype=L.RA_BF16, fmt=L.RA_MXFP4, k=_t(), v=NONE, q=NONE,
          km=_m(), vm=NO_MX, qm=NO_MX):
    return fn(ctypes.byref(L.ra_mx_desc(batch, heads, n_ref, head_dim, dtype, fmt)),
              ctypes.byref(L.ra_mx_args(k, v, q, km, vm, qm)), None)


@pytest.mark.parametrize("kw,status,msg", CASES)
def test_commit_and_read(kw, status, msg):
    for fn in (L.LIB.refadapt_mx_commit, L.LIB.refadapt_mx_read):
        st = _call(fn, **kw)
        assert st == status and msg in L.refadapt_last_error(), (st, L.refadapt_last_error())
        assert _call(fn, n_ref=0, k=NONE, km=NO_MX) == L.RA_OK
        assert fn(None, ctypes.byref(L.ra_mx_args()), None) == L.RA_EINVAL
        assert fn(ctypes.byref(L.ra_mx_desc()), None, None) == L.RA_EINVAL


def _attn(cache=None, ws=0x10000, ws_bytes=1 << 30, desc=None, args=None):
    d = dict(batch=1, heads=2, head_dim=128, n_ref=64, n_tgt=64, dtype=L.RA_BF16, scale=0.0, qset=L.RA_Q_TARGET,
             kvsrc=L.RA_KV_CACHE)
    d.update(desc or {})
    a = dict(q_tgt=_t(), k_tgt=_t(), v_tgt=_t(), o_tgt=_t(), workspace=ws, workspace_bytes=ws_bytes)
    a.update(args or {})
    c = dict(format=L.RA_MXFP4, k=_m(), v=_m())
    c.update(cache or {})
    st = L.LIB.refadapt_joint_attn_mx(ctypes.byref(L.ra_attn_desc(**d)), ctypes.byref(L.ra_attn_args(**a)),
                                      ctypes.byref(L.ra_mx_cache(**c)), None)
    return st, L.refadapt_last_error()


@pytest.mark.parametrize("kw,status,msg", [
    (dict(desc=dict(head_dim=96)), L.RA_EUNSUPPORTED, "head_dim"),
    (dict(desc=dict(n_tgt=0)), L.RA_EINVAL, "n_tgt"),
    (dict(desc=dict(kvsrc=L.RA_KV_FRESH)), L.RA_EUNSUPPORTED, "RA_KV_CACHE"),
    (dict(desc=dict(kvsrc=L.RA_KV_SEGMENTS)), L.RA_EUNSUPPORTED, "RA_KV_CACHE"),
    (dict(desc=dict(batch=70000)), L.RA_EUNSUPPORTED, "65535"),
    (dict(cache=dict(format=5)), L.RA_EINVAL, "format"),
    (dict(cache=dict(v=NO_MX)), L.RA_EINVAL, "v_mx"),
    (dict(cache=dict(k=_m(codes=0x1004))), L.RA_EUNSUPPORTED, "k_mx"),
    (dict(cache=dict(k=_m(ss=1 << 24))), L.RA_EUNSUPPORTED, "k_mx row strides"),
    (dict(cache=dict(v=_m(es=1 << 24))), L.RA_EUNSUPPORTED, "v_mx row strides"),
    (dict(args=dict(q_tgt=_t(0))), L.RA_EINVAL, "q_tgt"),
    (dict(args=dict(k_tgt=_t(ss=132))), L.RA_EUNSUPPORTED, "k_tgt"),
    (dict(args=dict(v_tgt=_t(ss=1 << 24))), L.RA_EUNSUPPORTED, "row stride"),
    (dict(args=dict(seg_mass=0x1000, n_seg=1)), L.RA_EUNSUPPORTED, "segments"),
    (dict(ws_bytes=16, desc=dict(n_tgt=4096)), L.RA_EWORKSPACE, "workspace"),
    (dict(ws=None, desc=dict(n_tgt=4096)), L.RA_EWORKSPACE, "workspace"),
    (dict(ws=0x10008, desc=dict(n_tgt=4096)), L.RA_EUNSUPPORTED, "workspace"),
    (dict(desc=dict(qset=L.RA_Q_ALL)), L.RA_EINVAL, "q_ref"),
    (dict(desc=dict(qset=L.RA_Q_ALL), cache=dict(q=_m())), L.RA_EINVAL, "o_ref"),
    (dict(desc=dict(kvsrc=L.RA_KV_DEVICE), args=dict(q_ref=_t(), k_ref=_t(), v_ref=_t(), o_ref=_t())), L.RA_EINVAL,
     "decision"),
    (dict(desc=dict(kvsrc=L.RA_KV_DEVICE), args=dict(q_ref=_t(), v_ref=_t(), o_ref=_t(), decision=0x1000)), L.RA_EINVAL,
     "k_ref"),
])
def test_attention(kw, status, msg):
    st, err = _attn(**kw)
    assert st == status and msg in err, (st, err)


def test_attention_null_blocks_and_workspace_sizes():
    d = L.ra_attn_desc(1, 2, 128, 64, 4096, L.RA_BF16, 0.0, L.RA_Q_ALL, L.RA_KV_CACHE)
    a = L.ra_attn_args()
    c = L.ra_mx_cache(L.RA_MXFP4)
    fn = L.LIB.refadapt_joint_attn_mx
    assert fn(ctypes.byref(d), ctypes.byref(a), None, None) == L.RA_EINVAL
    assert fn(None, ctypes.byref(a), ctypes.byref(c), None) == L.RA_EINVAL
    assert fn(ctypes.byref(d), None, ctypes.byref(c), None) == L.RA_EINVAL
    size = lambda q: L.refadapt_joint_attn_mx_workspace_size(d, L.RA_MXFP4, q)
    assert size(0) == 2 * 2 * 64 * 128 * 2 and size(1) == 3 * 2 * 64 * 128 * 2
    assert L.refadapt_joint_attn_mx_workspace_size(d, 7, 0) == 0
    d.kvsrc = L.RA_KV_FRESH
    assert size(0) == 0
    assert L.LIB.refadapt_joint_attn_mx_workspace_size(None, 0, 0) == 0
