"""Tensors that carry a tangent of forward-mode differentiation are refused: the library would leave it behind. (The
library's calls replaced by ones that do nothing; CPU tensors in place of the device's.)"""

import pytest
import torch
from torch.autograd import forward_ad

from paper_2609_32415_amd import ops

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.fixture
def made(monkeypatch):
    calls = []
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)  # a CPU tensor's device number
    monkeypatch.setattr(ops, "_stream", lambda: 0)
    monkeypatch.setattr(ops, "_on_gpu", lambda *a: None)
    for name in dir(ops.L):
        if name.startswith("refadapt_"):
            size = "size" in name
            monkeypatch.setattr(ops.L, name, lambda *a, size=size: 0 if size else calls.append(a))
    return calls


def _t(*shape, dtype=BF16):
    return torch.ones(shape, dtype=dtype)


def _mx():
    return ops.MxTensor(_t(1, 1, 4, 32, dtype=U8), _t(1, 1, 4, 2, dtype=U8), "mxfp4")


def _norm_tensors():
    return dict(x=_t(1, 4, 64), weight=_t(64), bias=_t(64), scale=_t(1, 64), shift=_t(1, 64))


def _grad_tensors():
    return dict(dy=_t(1, 4, 64), x=_t(1, 4, 64), stats=_t(1, 4, 2, dtype=F32), weight=_t(64), bias=_t(64),
                scale=_t(1, 64))


def _rope_tensors():
    freq, axis = ops.rope_frequencies((64,))
    return dict(q=_t(1, 2, 4, 64), k=_t(1, 2, 4, 64), pos=_t(4, 1, dtype=F32), freq=freq, axis=axis)


def _attn_tensors(**more):
    return dict({n: _t(1, 1, 4, 64) for n in ("q_tgt", "k_tgt", "v_tgt", "q_ref", "k_ref", "v_ref")}, **more)


def _two():
    return dict(q_cur=_t(1, 1, 4, 64), q_prev=_t(1, 1, 4, 64))


CALLS = {
    "layer_norm": (ops.layer_norm, _norm_tensors()),
    "layer_norm_mx": (lambda **t: ops.layer_norm_mx(fmt="mxfp4", **t), _norm_tensors()),
    "layer_norm_grad": (ops.layer_norm_grad, _grad_tensors()),
    "mx_linear": (lambda **t: ops.mx_linear(w=_mx(), **t), dict(x=_t(1, 4, 64), bias=_t(4))),
    "mx_linear of codes": (lambda **t: ops.mx_linear(_mx(), _mx(), **t), dict(bias=_t(4))),
    "mx_linear_grad": (lambda **t: ops.mx_linear_grad(w=_mx(), **t), dict(dy=_t(1, 3, 4))),
    "mx_commit": (lambda **t: ops.mx_commit(v_ref=None, k_mx=_mx(), v_mx=None, **t), dict(k_ref=_t(1, 1, 4, 64))),
    "rope": (ops.rope, _rope_tensors()),
    "joint_attn": (ops.joint_attn, _attn_tensors(k_cache=_t(1, 1, 4, 64), v_cache=_t(1, 1, 4, 64))),
    "joint_attn_mx": (lambda **t: ops.joint_attn_mx(k_mx=_mx(), v_mx=_mx(), **t), _attn_tensors()),
    "q_change": (lambda **t: ops.q_change(workspace=_t(64, dtype=U8), **t), _two()),
    "mass_mean": (ops.mass_mean, dict(mass=_t(1, 2, 4, dtype=F32))),
    "adjacent_mass_change": (ops.adjacent_mass_change, dict(mass_log=_t(3, 2, 1, dtype=F32))),
    "gate": (lambda **t: ops.gate(state=_t(4, dtype=I32), block=0, step=0, **t),
             dict(d_cur=_t(1, 1, dtype=F32), mass_prev=_t(1, 1, 4, dtype=F32), theta=_t(1, dtype=F32))),
    "q_change_gate": (lambda **t: ops.q_change_gate(state=_t(4, dtype=I32), block=0, step=0, workspace=_t(64, dtype=U8),
                                                    **t),
                      dict(_two(), mass_prev=_t(1, 1, 4, dtype=F32), theta=_t(1, dtype=F32))),
    "q_change_gate_noalloc": (lambda **t: ops.q_change_gate_noalloc(state=_t(4, dtype=I32), block=0, step=0, **t),
                              dict(_two(), mass_prev=_t(1, 1, 4, dtype=F32), theta=_t(1, dtype=F32))),
    "cache_commit": (lambda **t: ops.cache_commit(k_cache=_t(1, 1, 4, 64), v_cache=_t(1, 1, 4, 64), **t),
                     dict(k_ref=_t(1, 1, 4, 64), v_ref=_t(1, 1, 4, 64))),
    "kv_drift": (lambda **t: ops.kv_drift(workspace=_t(64, dtype=U8), **t),
                 {n: _t(1, 1, 4, 64) for n in ("k_cur", "k_base", "v_cur", "v_base")}),
    "output_impact": (lambda **t: ops.output_impact(workspace=_t(64, dtype=U8), **t),
                      dict(o_stale=_t(1, 1, 4, 64), o_fresh=_t(1, 1, 4, 64))),
}
CASES = [(name, n) for name, (_, tensors) in CALLS.items() for n, t in tensors.items() if t.is_floating_point()]


@pytest.mark.parametrize("name,which", CASES)
def test_refused(made, name, which):
    call, tensors = CALLS[name]
    call(**tensors)
    n = len(made)
    assert n
    with forward_ad.dual_level():
        call(**tensors)  # none carries one
        assert len(made) == 2 * n
        dual = forward_ad.make_dual(tensors[which], torch.ones_like(tensors[which]))
        with pytest.raises(ValueError, match="tangent"):
            call(**{**tensors, which: dual})
        with torch.no_grad(), pytest.raises(ValueError, match="tangent"):  # it does not switch these off
            call(**{**tensors, which: dual})
    assert len(made) == 2 * n
    call(**tensors)


def test_beside_a_recorded_call(made):
    """A parameter that requires grad, and rows that carry a tangent."""
    with forward_ad.dual_level():
        x = forward_ad.make_dual(_t(1, 4, 64), _t(1, 4, 64))
        with pytest.raises((ValueError, RuntimeError)):
            ops.layer_norm(x, _t(64).requires_grad_())
        with pytest.raises((ValueError, RuntimeError)):
            ops.mx_linear(x, _mx(), _t(4).requires_grad_())
