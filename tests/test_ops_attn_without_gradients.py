"""The attention has no gradients: a backward pass that reaches it raises, where its inputs would have been left out in
silence. (The library's calls replaced by ones that do nothing; CPU tensors in place of the device's.)"""

import pytest
import torch

from paper_2609_32415_amd import ops


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)  # a CPU tensor's device number
    monkeypatch.setattr(ops, "_stream", lambda: 0)
    monkeypatch.setattr(ops, "_on_gpu", lambda *a: None)
    for name in dir(ops.L):
        if name.startswith("refadapt_"):
            monkeypatch.setattr(ops.L, name, lambda *a: 0)


def _heads():
    return torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16)


def _inputs():
    return {n: _heads() for n in ("q_tgt", "k_tgt", "v_tgt", "q_ref", "k_ref", "v_ref")}


def _mx():
    return ops.MxTensor(*(torch.zeros((1, 1, 4, n), dtype=torch.uint8) for n in (32, 2)), "mxfp4")


def _joint_attn_mx(**kw):
    return ops.joint_attn_mx(k_mx=_mx(), v_mx=_mx(), **kw)


CALLS = {"joint_attn": ops.joint_attn, "joint_attn_mx": _joint_attn_mx}


@pytest.mark.parametrize("which", list(_inputs()))
@pytest.mark.parametrize("name", CALLS)
def test_a_backward_pass_raises(name, which):
    t = _inputs()
    t[which].requires_grad_()
    out = CALLS[name](**t, qset="all", lse=True, ref_mass_refq=True)
    hidden = torch.zeros((1, 1, 4, 64), requires_grad=True)
    for result in (out.o_tgt, out.o_ref, out.ref_mass, out.lse, out.ref_mass_refq):
        assert result.requires_grad
        with pytest.raises(NotImplementedError, match=f"{name} has no gradients"):
            (hidden.sum() + result.sum()).backward()


@pytest.mark.parametrize("name", CALLS)
def test_given_buffers_stay_as_they_are(name):
    t = _inputs()
    t["q_tgt"].requires_grad_()
    o, mass = _heads(), torch.zeros((1, 1, 4))
    for _ in range(2):
        out = CALLS[name](**t, o_tgt=o, ref_mass=mass)
        assert not o.requires_grad and not mass.requires_grad and out.o_tgt.data_ptr() == o.data_ptr()
        with pytest.raises(NotImplementedError):
            out.o_tgt.sum().backward()


@pytest.mark.parametrize("name", CALLS)
def test_without_recording(name):
    t = _inputs()
    o = _heads()
    assert CALLS[name](**t, o_tgt=o).o_tgt is o
    t["v_tgt"].requires_grad_()
    with torch.no_grad():
        out = CALLS[name](**t, o_tgt=o)
        assert out.o_tgt is o and not out.ref_mass.requires_grad
    with torch.inference_mode():
        assert CALLS[name](**t).o_tgt.shape == o.shape
