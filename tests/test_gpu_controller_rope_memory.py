"""The controller's turned Q and K: the same trajectory as from inputs that were turned before, and memory that does not
grow with the captured steps."""

import gc

import numpy as np
import pytest
import torch

from gpu_helpers import dev
from paper_2609_32415_amd import ops, synth
from paper_2609_32415_amd.controller import Controller, Rope, Sidecar, StepGraphs

pytestmark = pytest.mark.gpu

ROLES = ("q_tgt", "k_tgt", "v_tgt", "q_ref", "k_ref", "v_ref")


def _rope(w):
    pos = lambda n, t: torch.from_numpy(np.stack((np.full(n, t), np.arange(n) // 16, np.arange(n) % 16), 1)
                                        .astype(np.int32)).to("cuda:0")
    return Rope(*ops.rope_frequencies((16, 56, 56)), pos(w.n_ref, 1), pos(w.n_tgt, 0))


def _controller(w, **kw):
    return Controller(w.n_blocks, w.n_steps, w.batch, w.heads, w.n_ref, w.n_tgt, w.head_dim, 0.08, device="cuda:0", **kw)


@pytest.mark.parametrize("cue,fmt,sidecar", [("consecutive", None, False), ("consecutive", "mxfp8", True),
                                             ("anchor", "mxfp4", False)])
def test_same_as_inputs_turned_before(cue, fmt, sidecar):
    w = synth.workload("sweep", heads=2, n_ref=70, n_tgt=90, n_blocks=3, n_steps=5, seed=5)
    trajs = [synth.Trajectory(w, b, ref_sigma=lambda t, b=b: synth.sweep_ref_drift(b, w.n_blocks),
                              tgt_sigma=lambda t: synth.sweep_tgt_drift(t, w.n_steps)) for b in range(w.n_blocks)]
    xs = {(t, b): {n: dev(v, "bf16") for n, v in trajs[b].step_tensors(t).items() if n in ROLES}
          for t in range(w.n_steps) for b in range(w.n_blocks)}
    rope = _rope(w)
    probes = lambda: Sidecar(w.n_blocks, w.n_steps, w.batch, w.heads, w.n_ref, w.n_tgt, w.head_dim) if sidecar else None
    want, got = [_controller(w, cue=cue, cache_format=fmt, rope=r, sidecar=probes()) for r in (None, rope)]
    steps = []
    for t in range(w.n_steps):
        if t == 2:  # inputs that come out of a recorded graph
            xs[(t, 0)]["q_tgt"].requires_grad_()
        want.step(t, [rope.turned(xs[(t, b)]) for b in range(w.n_blocks)])
        got.step(t, [xs[(t, b)] for b in range(w.n_blocks)])
        torch.cuda.synchronize()
        steps.append([o.clone() for o in want.o_tgt + want.o_ref] + [want.recorded_mass(b).clone() for b in range(w.n_blocks)])
        mine = got.o_tgt + got.o_ref + [got.recorded_mass(b) for b in range(w.n_blocks)]
        assert all(torch.equal(a, b) for a, b in zip(steps[-1], mine)), t
    assert torch.equal(want.decisions, got.decisions) and torch.equal(want.scores, got.scores)
    if sidecar:
        for n in ("e_kv", "rho_k", "rho_v", "impact", "m_cached"):
            assert torch.equal(getattr(want.sidecar, n).nan_to_num(7.0), getattr(got.sidecar, n).nan_to_num(7.0)), n
        return
    # captured, an odd number of steps, twice over
    ctl = _controller(w, cue=cue, cache_format=fmt, rope=rope)
    graphs = StepGraphs(ctl, lambda: [{n: torch.empty_like(v) for n, v in xs[(0, b)].items()} for b in range(w.n_blocks)])
    for rep in range(2):
        for t in range(w.n_steps):
            for b, buf in enumerate(graphs.inputs(t)):
                for n, v in buf.items():
                    v.copy_(xs[(t, b)][n].detach())
            torch.cuda.synchronize()
            graphs.replay(t)
            torch.cuda.synchronize()
            n = 2 * w.n_blocks
            assert all(torch.equal(a, b) for a, b in zip(steps[t][:n // 2], ctl.o_tgt)), (rep, t)
            assert all(torch.equal(a, graphs.recorded_mass(t, b)) for b, a in enumerate(steps[t][n:])), (rep, t)
        # (step 0 has nothing to compare with: its scores come of whatever mass is there, and decide nothing)
        assert torch.equal(ctl.decisions, want.decisions) and torch.equal(ctl.scores[1:], want.scores[1:])


def test_captured_steps_keep_no_memory():
    """What the allocator holds for the graphs of two steps and of six. A block's four turned tensors are 8 MiB each."""
    def held(n_steps):
        w = synth.workload("sweep", heads=8, n_ref=4096, n_tgt=4096, n_blocks=2, n_steps=n_steps, seed=1)
        gc.collect()
        torch.cuda.empty_cache()
        before = torch.cuda.memory_reserved()
        ctl = _controller(w, rope=_rope(w), cache_format="mxfp4")
        new = lambda: [{n: torch.zeros(ctl.shape_t if n.endswith("tgt") else ctl.shape_r, dtype=torch.bfloat16,
                                       device="cuda:0") for n in ROLES} for _ in range(w.n_blocks)]
        graphs = StepGraphs(ctl, new)
        gc.collect()
        torch.cuda.empty_cache()
        n = torch.cuda.memory_reserved() - before
        del graphs, ctl
        return n

    held(2)
    a, b = held(2), held(6)
    assert b - a < (8 << 20), (a, b)
