"""Keys without weight, and keys that are no numbers, in joint attention of both types: whole query tiles, key ranges
and their merge, reference segments.

A key of scores of -inf, or far below the rest, has no part in any output: they are those of the fp64 formula. Tolerance
of a bf16 output: its own rounding (2^-8 of the value), the probabilities' (2^-8 each, of the numerator and of the sum
that divides) and fp32 scores (below 2^-10 in the exponent), of the attention-weighted mean of |v|; the path's bars
otherwise. A NaN key is in every sum over its side: o, the masses and the log-sum-exp of all keys are NaN, and that of
the reference where the key is one of it.
"""

import numpy as np
import pytest
import torch

from gpu_helpers import MASS_TOL, O_TOL, TORCH_DTYPE, host, max_abs
from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu

SIZES = [(330, 290), (2000, 40), (70, 600)]  # the reference's tiles, the target's, each ragged
FINE = 1e-3  # log-sum-exp


def _inputs(dtype, d, n_ref, n_tgt):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(n_ref + n_tgt + d)
    t = lambda n: torch.randn((1, 2, n, d), generator=g, device="cuda:0").to(TORCH_DTYPE[dtype])
    x = {r + "_" + s: t(n) for s, n in (("tgt", n_tgt), ("ref", n_ref)) for r in "qkv"}
    x["q_tgt"][..., 0] = x["q_ref"][..., 0] = 1.0
    return x


def _run(x, workspace, n_seg=0, **kw):
    ws = ops.attn_workspace(x["q_tgt"], x["k_ref"].shape[2], qset="all", n_seg_mass=n_seg) if workspace else False
    return ops.joint_attn(x["q_tgt"], x["k_tgt"], x["v_tgt"], q_ref=x["q_ref"], k_ref=x["k_ref"], v_ref=x["v_ref"],
                          qset="all", lse=True, ref_mass_refq=True, workspace=ws, **kw)


def _lse(s):
    top = s.max(-1)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(top), top + np.log(np.exp(s - top[..., None]).sum(-1)), top)


def _gone(n_ref, n_tgt):
    r, t = np.zeros(n_ref, bool), np.zeros(n_tgt, bool)
    some = np.random.default_rng(1)
    yield "first reference tile", (np.arange(n_ref) < min(64, n_ref - 1)), t
    yield "half of the reference", (np.arange(n_ref) < n_ref // 2), t
    yield "all but the last reference key", (np.arange(n_ref) < n_ref - 1), t
    yield "the reference", ~r, t
    yield "the target", r, ~t
    yield "scattered", some.random(n_ref) < 0.7, some.random(n_tgt) < 0.7
    yield "all but the last target key", ~r, (np.arange(n_tgt) < n_tgt - 1)


PATHS = [("bf16", False), ("bf16", True), ("f32", False)]
PATH_IDS = ["bf16 whole", "bf16 ranges", "f32"]


def _close(o, want, av, dtype):
    tol = O_TOL["f32"]
    if dtype == "bf16":
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -10) * (av + np.abs(want)) + 1e-6
    return (np.abs(host(o) - want) <= tol).all()


@pytest.mark.parametrize("dtype,workspace", PATHS, ids=PATH_IDS)
@pytest.mark.parametrize("n_ref,n_tgt", SIZES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("score", [float("-inf"), -2.0 ** 30])
def test_keys_without_weight(score, dtype, d, n_ref, n_tgt, workspace):
    base = _inputs(dtype, d, n_ref, n_tgt)
    for what, gr, gt in _gone(n_ref, n_tgt):
        x = {k: v.clone() for k, v in base.items()}
        x["k_ref"][:, :, torch.from_numpy(gr).to("cuda:0"), 0] = score
        x["k_tgt"][:, :, torch.from_numpy(gt).to("cuda:0"), 0] = score
        print(score, dtype, d, n_ref, n_tgt, workspace, what, flush=True)
        r = _run(x, workspace)
        # without mass and log-sum-exp: the same outputs
        bare = ops.joint_attn(x["q_tgt"], x["k_tgt"], x["v_tgt"], q_ref=x["q_ref"], k_ref=x["k_ref"], v_ref=x["v_ref"],
                              qset="all", ref_mass=False, workspace=None if workspace else False)
        torch.cuda.synchronize()
        h = {k: host(v) for k, v in x.items()}
        k = np.concatenate((h["k_ref"], h["k_tgt"]), 2)
        v = np.concatenate((h["v_ref"], h["v_tgt"]), 2)
        for q, o, mass, lse in ((h["q_tgt"], r.o_tgt, r.ref_mass, r.lse), (h["q_ref"], r.o_ref, r.ref_mass_refq, None)):
            s = q @ k.swapaxes(2, 3) / np.sqrt(d)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            assert _close(o, p @ v, p @ np.abs(v), dtype), what
            assert max_abs(host(mass), p[..., :n_ref].sum(-1)) <= MASS_TOL[dtype], what
            if lse is not None:
                w = np.stack((_lse(s[..., :n_ref]), _lse(s)), -1)
                got, fin = host(lse), np.isfinite(w)
                assert np.array_equal(got[~fin], w[~fin]), what
                assert (np.abs(got[fin] - w[fin]) <= FINE + 2.0 ** -21 * np.abs(w[fin])).all(), what
        assert torch.equal(bare.o_tgt, r.o_tgt) and torch.equal(bare.o_ref, r.o_ref), what


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "ranges"])
@pytest.mark.parametrize("d", [64, 128])
def test_segments_without_weight(d, workspace):
    n_ref, n_tgt, ends = 700, 290, [128, 320, 640, 700]
    x = _inputs("bf16", d, n_ref, n_tgt)
    gr = np.zeros(n_ref, bool)
    gr[:128] = gr[330:640] = True  # the first segment and most of the third
    x["k_ref"][:, :, torch.from_numpy(gr).to("cuda:0"), 0] = float("-inf")
    r = _run(x, workspace, n_seg=4, seg_end=ends, seg_mass=True)
    torch.cuda.synchronize()
    q, k = host(x["q_tgt"]), np.concatenate((host(x["k_ref"]), host(x["k_tgt"])), 2)
    s = q @ k.swapaxes(2, 3) / np.sqrt(d)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    parts = np.split(p, ends, -1)[:4]
    want = np.stack([a.sum(-1) for a in parts], -1)
    got = host(r.seg_mass)
    assert max_abs(got, want) <= MASS_TOL["bf16"] and (got[..., 0] == 0).all()
    assert max_abs(host(r.ref_mass), want.sum(-1)) <= MASS_TOL["bf16"]
    v = np.concatenate((host(x["v_ref"]), host(x["v_tgt"])), 2)
    assert _close(r.o_tgt, p @ v, p @ np.abs(v), "bf16")


@pytest.mark.parametrize("dtype,workspace", PATHS, ids=PATH_IDS)
@pytest.mark.parametrize("n_ref,n_tgt", SIZES)
@pytest.mark.parametrize("d", [64, 128])
def test_nan_keys(dtype, d, n_ref, n_tgt, workspace):
    x = _inputs(dtype, d, n_ref, n_tgt)
    clean = _run(x, workspace)
    for side, n in (("ref", n_ref), ("tgt", n_tgt)):
        for row in (0, n // 2, n - 1):
            k = x["k_" + side]
            old = k[0, 1, row, 5].clone()
            k[0, 1, row, 5] = float("nan")
            r = _run(x, workspace)
            k[0, 1, row, 5] = old
            torch.cuda.synchronize()
            print(dtype, d, n_ref, n_tgt, workspace, side, row, flush=True)
            for t in (r.o_tgt, r.o_ref, r.ref_mass, r.ref_mass_refq, r.lse[..., 1]):
                assert torch.isnan(t[0, 1]).all(), (side, row)
            if side == "ref":
                assert torch.isnan(r.lse[0, 1, :, 0]).all(), row
            else:  # formed before the target's keys, but by another tile's maximum in a range with the NaN
                assert max_abs(host(r.lse[0, 1, :, 0]), host(clean.lse[0, 1, :, 0])) <= FINE, row
            for a, b in ((r.o_tgt, clean.o_tgt), (r.o_ref, clean.o_ref), (r.ref_mass, clean.ref_mass),
                         (r.lse, clean.lse), (r.ref_mass_refq, clean.ref_mass_refq)):
                assert torch.equal(a[0, 0], b[0, 0]), (side, row)


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "ranges"])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_keys_of_segments(d, workspace):
    """The NaN is in the sum that every segment's mass is a share of."""
    n_ref, n_tgt, ends = 700, 290, [128, 320, 640, 700]
    x = _inputs("bf16", d, n_ref, n_tgt)
    for row in (3, 400, 699):
        old = x["k_ref"][0, 0, row, 5].clone()
        x["k_ref"][0, 0, row, 5] = float("nan")
        r = _run(x, workspace, n_seg=4, seg_end=ends, seg_mass=True)
        x["k_ref"][0, 0, row, 5] = old
        torch.cuda.synchronize()
        assert torch.isnan(r.seg_mass[0, 0]).all() and torch.isnan(r.ref_mass[0, 0]).all() and \
            torch.isnan(r.o_tgt[0, 0]).all(), row
        assert torch.isfinite(r.seg_mass[0, 1]).all() and torch.isfinite(r.o_tgt[0, 1]).all(), row
