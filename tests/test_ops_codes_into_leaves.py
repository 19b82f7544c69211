"""A projection of codes is not written into a tensor that requires grad while gradients are recorded, as one of plain
rows is not. (The library's calls replaced by ones that do nothing; CPU tensors in place of the device's.)"""

import pytest
import torch

from paper_2609_32415_amd import ops


@pytest.mark.parametrize("codes", [False, True])
def test_refused(codes, monkeypatch):
    made = []
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)  # a CPU tensor's device number
    monkeypatch.setattr(ops, "_stream", lambda: 0)
    monkeypatch.setattr(ops, "_on_gpu", lambda *a: None)
    monkeypatch.setattr(ops.L, "refadapt_mx_linear_packed", lambda *a: made.append(a))
    mx = lambda n: ops.MxTensor(*(torch.zeros((1, 1, n, k), dtype=torch.uint8) for k in (32, 2)), "mxfp4")
    x, w = mx(4) if codes else torch.zeros((1, 4, 64), dtype=torch.bfloat16), mx(8)
    leaf = torch.zeros((1, 4, 8), dtype=torch.bfloat16, requires_grad=True)
    with pytest.raises(ValueError, match="out cannot be given"):
        ops.mx_linear(x, w, out=leaf)
    assert not made
    with torch.no_grad():
        assert ops.mx_linear(x, w, out=leaf) is leaf
    assert ops.mx_linear(x, w, out=leaf.detach()).requires_grad is False
    assert len(made) == 2
