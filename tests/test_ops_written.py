"""What the wrappers write into a caller's tensors counts as a change in place (the library's calls replaced by ones
that do nothing; CPU tensors in place of the device's)."""

import pytest
import torch

from paper_2609_32415_amd import ops

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)  # a CPU tensor's device number
    monkeypatch.setattr(ops, "_stream", lambda: 0)
    monkeypatch.setattr(ops, "_on_gpu", lambda *a: None)
    for name in dir(ops.L):
        if name.startswith("refadapt_"):
            monkeypatch.setattr(ops.L, name, lambda *a: 0)


def _t(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype)


def _mx(h=1, n=4):
    return ops.MxTensor(_t(1, h, n, 32, dtype=U8), _t(1, h, n, 2, dtype=U8), "mxfp4")


def _heads():
    return _t(1, 2, 4, 64)


STATS = dict(mass_prev=_t(1, 2, 4, dtype=F32), theta=_t(4, dtype=F32), block=0, step=0)
MASSES = dict(ref_mass=(1, 2, 4), lse=(1, 2, 4, 2), ref_mass_refq=(1, 2, 4))


def _calls():
    yield "layer_norm", lambda o: ops.layer_norm(_t(1, 4, 64), out=o[0]), [_t(1, 4, 64)]
    m = _mx()
    yield "layer_norm_mx", lambda o: ops.layer_norm_mx(_t(1, 4, 64), "mxfp4", out=m), [m.codes, m.scales]
    yield "mx_linear", lambda o: ops.mx_linear(_t(1, 4, 64), _mx(), out=o[0]), [_t(1, 4, 4)]
    yield "mx_linear of codes", lambda o: ops.mx_linear(_mx(), _mx(), out=o[0]), [_t(1, 4, 4)]
    caches = [_mx(2) for _ in range(3)]
    yield "mx_commit", lambda o: ops.mx_commit(_heads(), _heads(), caches[0], caches[1], age=o[-1], q_ref=_heads(),
                                               q_mx=caches[2]), \
        [*(t for c in caches for t in (c.codes, c.scales)), _t(1, dtype=I32)]
    yield "mx_read", lambda o: ops.mx_read(_mx(2), _mx(2), _mx(2), k_out=o[0], v_out=o[1], q_out=o[2]), \
        [_heads() for _ in range(3)]
    freq, axis = ops.rope_frequencies((64,))
    yield "rope", lambda o: ops.rope(_heads(), _heads(), pos=_t(4, 1, dtype=I32), freq=freq, axis=axis, q_out=o[0],
                                     k_out=o[1]), [_heads(), _heads()]
    masses = lambda: [_t(*s, dtype=F32) for s in MASSES.values()]
    yield "joint_attn", lambda o: ops.joint_attn(
        *(_heads() for _ in range(3)), q_ref=_heads(), k_ref=_heads(), v_ref=_heads(), qset="all", o_tgt=o[0],
        o_ref=o[1], **dict(zip(MASSES, o[2:])), workspace=False), [_heads(), _heads(), *masses()]
    yield "joint_attn segments", lambda o: ops.joint_attn(
        *(_heads() for _ in range(3)), k_ref=_heads(), v_ref=_heads(), seg_end=[4], o_tgt=o[0], seg_mass=o[1],
        workspace=False), [_heads(), _t(1, 2, 4, 1, dtype=F32)]
    yield "joint_attn_mx", lambda o: ops.joint_attn_mx(
        *(_heads() for _ in range(3)), k_mx=_mx(2), v_mx=_mx(2), q_ref=_heads(), qset="all", o_tgt=o[0], o_ref=o[1],
        **dict(zip(MASSES, o[2:]))), [_heads(), _heads(), *masses()]
    yield "cache_commit", lambda o: ops.cache_commit(_heads(), _heads(), o[0], o[1], age=o[3], q_ref=_heads(),
                                                     q_cache=o[2]), [*(_heads() for _ in range(3)), _t(1, dtype=I32)]
    ws = _t(64, dtype=U8)
    yield "q_change", lambda o: ops.q_change(_heads(), _heads(), out=o[0], workspace=ws), [_t(1, 2, dtype=F32)]
    yield "gate", lambda o: ops.gate(_t(1, 2, dtype=F32), state=o[0], decision_out=o[1], score_out=o[2], **STATS), \
        [_t(4, dtype=I32), _t(1, dtype=I32), _t(3, dtype=F32)]
    for name, kw in (("q_change_gate", dict(workspace=ws)), ("q_change_gate_noalloc", {})):
        yield name, lambda o, name=name, kw=kw: getattr(ops, name)(
            _heads(), _heads(), state=o[0], decision_out=o[1], score_out=o[2], d_out=o[3], **STATS, **kw), \
            [_t(4, dtype=I32), _t(1, dtype=I32), _t(3, dtype=F32), _t(1, 2, dtype=F32)]
    two = lambda n: [_t(1, 2, dtype=F32) for _ in range(n)]
    yield "kv_drift", lambda o: ops.kv_drift(*(_heads() for _ in range(4)), d_k=o[0], d_v=o[1], e_kv=o[2],
                                             workspace=ws), two(3)
    yield "drift_log_ratio", lambda o: ops.drift_log_ratio(*(_heads() for _ in range(4)), d_ref=o[0], d_tgt=o[1],
                                                           rho=o[2], workspace=ws), two(3)
    yield "output_impact", lambda o: ops.output_impact(_heads(), _heads(), out=o[0], workspace=ws), two(1)
    yield "mass_mean", lambda o: ops.mass_mean(_t(1, 2, 4, dtype=F32), out=o[0]), two(1)
    yield "adjacent_mass_change", lambda o: ops.adjacent_mass_change(_t(3, 2, 1, dtype=F32), out=o[0]), \
        [_t(2, dtype=F32)]


CALLS = {name: (call, outs) for name, call, outs in _calls()}


@pytest.mark.parametrize("name", CALLS)
def test_writes_are_counted(name):
    call, outs = CALLS[name]
    before = [t._version for t in outs]
    call(outs)
    assert all(t._version > b for t, b in zip(outs, before))


@pytest.mark.parametrize("name", CALLS)
def test_in_inference_mode(name):
    with torch.inference_mode():
        call, outs = next((c, o) for n, c, o in _calls() if n == name)
        call(outs)


def test_a_saved_tensor_that_was_written():
    """An input that a recorded call saved, and weights, written by the wrappers before the backward pass."""
    weight = torch.ones(64, dtype=BF16, requires_grad=True)
    x, w = _t(1, 4, 64), _mx()
    y = ops.layer_norm(x, weight)
    with torch.no_grad():
        ops.layer_norm(x, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(torch.ones_like(y))
    y = ops.mx_linear(_t(1, 4, 64).requires_grad_(), w)
    ops.mx_commit(_t(1, 1, 4, 64), None, w, None)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(torch.ones_like(y))
    buf = _t(1, 4, 4).requires_grad_()
    z = buf.detach()
    y = buf.exp().sum() + (buf * z).sum()
    ops.mx_linear(_t(1, 4, 64), w, out=z)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
