"""Joint attention over a quantised reference cache against the fp64 oracle over the values that the cache stands for.

Tolerance of an output of bf16 attention, with A|v| the attention-weighted mean of |v|: its own rounding (2^-8 of the
value); the probabilities' rounding to bf16 (2^-8 each, of the numerator and of the sum that divides: 2^-8 (A|v| + |o|));
fp32 scores, below 2^-10 in the exponent at these sizes: 2^-10 (A|v| + |o|). fp32: sums of up to n terms, held to the
bar of the fp32 path. Masses: the bars of the paths.
"""

import numpy as np
import pytest
import torch

from gpu_helpers import MASS_TOL, O_TOL, TORCH_DTYPE, host
from oracle import joint_attention, mx as oracle_mx
from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu


def _inputs(seed, B, H, n_ref, n_tgt, d, dtype, fmt, layout="bhsd", peak=1.0):
    rng = np.random.default_rng(seed)

    def t(n, amp=1.0):
        x = torch.from_numpy((amp * rng.standard_normal((B, H, n, d))).astype(np.float32)).to(TORCH_DTYPE[dtype])
        x = x.to("cuda:0")
        return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if layout == "bshd" else x

    x = {"q_tgt": t(n_tgt, peak), "k_tgt": t(n_tgt), "v_tgt": t(n_tgt), "q_ref": t(n_ref, peak), "k_ref": t(n_ref),
         "v_ref": t(n_ref)}
    c = {n: ops.mx_tensor((B, H, n_ref, d), fmt, "cuda:0") for n in "kvq"}
    if n_ref:
        ops.mx_commit(t(n_ref), t(n_ref), c["k"], c["v"], q_ref=t(n_ref, peak), q_mx=c["q"])
    vals = {n: oracle_mx.values(m.codes.cpu().numpy(), m.scales.cpu().numpy(), fmt) for n, m in c.items()}
    return x, c, vals


def _check_rows(o, mass, lse, q, kr, vr, x, dtype, scale=None):
    ky, vy = host(x["k_tgt"]), host(x["v_tgt"])
    ref = joint_attention(q, kr, vr, ky, vy, scale)
    err = np.abs(host(o) - ref["o"])
    if dtype == "bf16":
        av = joint_attention(q, kr, np.abs(vr), ky, np.abs(vy), scale)["o"]
        tol = 2.0 ** -8 * np.abs(ref["o"]) + (2.0 ** -8 + 2.0 ** -10) * (av + np.abs(ref["o"])) + 1e-6
    else:
        tol = O_TOL["f32"]
    assert (err <= tol).all(), float((err - tol).max())
    if mass is not None:
        assert np.abs(host(mass) - ref["ref_mass"]).max() <= MASS_TOL[dtype]
    if lse is not None:
        want = np.stack((ref["lse_ref"], ref["lse_all"]), -1)
        got = host(lse)
        fin = np.isfinite(want)
        assert np.array_equal(got[~fin], want[~fin]) and np.abs(got[fin] - want[fin]).max() <= 1e-3


SIZES = [
    # B, H, n_ref, n_tgt, d
    (1, 1, 1, 1, 64), (1, 2, 31, 1, 128), (2, 1, 33, 2, 64), (1, 3, 64, 17, 128), (1, 2, 65, 32, 128),
    (1, 2, 300, 33, 64), (2, 2, 129, 64, 128), (1, 4, 1000, 61, 128), (1, 2, 511, 65, 64), (1, 3, 257, 130, 128),
    (1, 2, 700, 257, 128), (1, 1, 4352, 5, 128), (1, 2, 5000, 40, 64), (3, 5, 96, 48, 64),
    (1, 2, 130, 1024, 64), (1, 1, 90, 1025, 128), (2, 30, 40, 300, 64), (3, 100, 33, 3, 64),
]


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,n_ref,n_tgt,d", SIZES)
def test_target_queries(fmt, dtype, B, H, n_ref, n_tgt, d):
    x, c, vals = _inputs(n_ref + n_tgt, B, H, n_ref, n_tgt, d, dtype, fmt, layout="bshd" if n_tgt % 2 else "bhsd")
    print("attn_mx", fmt, dtype, B, H, n_ref, n_tgt, d, flush=True)
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], lse=True)
    torch.cuda.synchronize()
    _check_rows(r.o_tgt, r.ref_mass, r.lse, host(x["q_tgt"]), vals["k"], vals["v"], x, dtype)
    # without mass and log-sum-exp, and again: the same outputs
    r2 = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], ref_mass=False)
    torch.cuda.synchronize()
    assert r2.ref_mass is None and torch.equal(r.o_tgt, r2.o_tgt)


@pytest.mark.parametrize("fmt,dtype,n_ref,n_tgt,d", [("mxfp4", "bf16", 333, 100, 128), ("mxfp8", "bf16", 190, 30, 64),
                                                     ("mxfp8", "f32", 129, 40, 64)])
def test_all_queries_with_and_without_cached_queries(fmt, dtype, n_ref, n_tgt, d):
    x, c, vals = _inputs(7, 1, 3, n_ref, n_tgt, d, dtype, fmt)
    for cached in (True, False):
        print("attn_mx all queries", fmt, dtype, cached, flush=True)
        kw = dict(q_mx=c["q"]) if cached else dict(q_ref=x["q_ref"])
        r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], qset="all", lse=True,
                              ref_mass_refq=True, **kw)
        torch.cuda.synchronize()
        _check_rows(r.o_tgt, r.ref_mass, r.lse, host(x["q_tgt"]), vals["k"], vals["v"], x, dtype)
        _check_rows(r.o_ref, r.ref_mass_refq, None, vals["q"] if cached else host(x["q_ref"]), vals["k"], vals["v"], x,
                    dtype)


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("decision", [ops.REUSE, ops.REACTIVATE, ops.COMPUTE])
def test_device_decisions(fmt, decision):
    """REUSE: target rows over the cache, o_ref untouched; REACTIVATE: all rows, the cached queries; COMPUTE: all
    rows, fresh K, V and queries."""
    x, c, vals = _inputs(11, 2, 2, 150, 70, 128, "bf16", fmt)
    word = torch.tensor([decision], dtype=torch.int32, device="cuda:0")
    o_ref = torch.full((2, 2, 150, 128), 5.0, dtype=torch.bfloat16, device="cuda:0")
    print("attn_mx device", fmt, decision, flush=True)
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], q_mx=c["q"], q_ref=x["q_ref"],
                          k_ref=x["k_ref"], v_ref=x["v_ref"], kvsrc="device", decision=word, o_ref=o_ref)
    torch.cuda.synchronize()
    kr, vr = (host(x["k_ref"]), host(x["v_ref"])) if decision == ops.COMPUTE else (vals["k"], vals["v"])
    _check_rows(r.o_tgt, r.ref_mass, None, host(x["q_tgt"]), kr, vr, x, "bf16")
    if decision == ops.REUSE:
        assert (o_ref == 5).all()
    else:
        _check_rows(r.o_ref, None, None, host(x["q_ref"]) if decision == ops.COMPUTE else vals["q"], kr, vr, x, "bf16")


def test_scores_far_apart_and_given_scale():
    """A large scale and peaked queries: the running maximum moves, most probabilities vanish."""
    for n_tgt in (3, 60, 300):
        x, c, vals = _inputs(13, 1, 2, 900, n_tgt, 128, "bf16", "mxfp8", peak=4.0)
        r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], scale=0.2)
        torch.cuda.synchronize()
        _check_rows(r.o_tgt, r.ref_mass, None, host(x["q_tgt"]), vals["k"], vals["v"], x, "bf16", 0.2)


@pytest.mark.parametrize("n_tgt", [1, 40, 200])
def test_nan_block_reaches_the_rows_that_see_it_and_no_reference(n_tgt):
    x, c, vals = _inputs(17, 1, 2, 70, n_tgt, 64, "bf16", "mxfp4")
    c["v"].scales[0, 1, 69, 1] = 255
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"])
    torch.cuda.synchronize()
    assert torch.isfinite(r.o_tgt[0, 0]).all() and torch.isfinite(r.o_tgt[0, 1, :, :32]).all()
    assert torch.isnan(r.o_tgt[0, 1, :, 32:]).all() and torch.isfinite(r.ref_mass).all()
    # a NaN block of K: every row of its head, no other
    c["k"].scales[0, 0, 3, 0] = 255
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"])
    torch.cuda.synchronize()
    assert torch.isnan(r.o_tgt[0, 0]).all() and torch.isnan(r.ref_mass[0, 0]).all()
    assert torch.isfinite(r.o_tgt[0, 1, :, :32]).all() and torch.isfinite(r.ref_mass[0, 1]).all()
    # an empty cache: plain self-attention
    empty = ops.mx_tensor((1, 2, 0, 64), "mxfp4", "cuda:0")
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=empty, v_mx=empty, lse=True)
    torch.cuda.synchronize()
    z = np.zeros((1, 2, 0, 64))
    _check_rows(r.o_tgt, r.ref_mass, r.lse, host(x["q_tgt"]), z, z, x, "bf16")
    assert (r.ref_mass == 0).all()


@pytest.mark.parametrize("n_tgt", [9, 200])
def test_rows_of_a_longer_cache_and_nothing_written_past_the_outputs(n_tgt):
    x, c, vals = _inputs(19, 2, 3, 130, n_tgt, 128, "bf16", "mxfp4")
    n = 75
    o = torch.full((2, 3, n_tgt + 2, 128), 9.0, dtype=torch.bfloat16, device="cuda:0")
    need = ops.attn_mx_workspace(x["q_tgt"], n, "mxfp4").numel()
    ws = torch.full((need + 64,), 77, dtype=torch.uint8, device="cuda:0")
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"].rows(n), v_mx=c["v"].rows(n),
                          o_tgt=o[:, :, 1:n_tgt + 1], workspace=ws[:need] if need else ws)
    torch.cuda.synchronize()
    _check_rows(r.o_tgt, r.ref_mass, None, host(x["q_tgt"]), vals["k"][:, :, :n], vals["v"][:, :, :n], x, "bf16")
    assert (o[:, :, 0] == 9).all() and (o[:, :, -1] == 9).all() and (ws[need:] == 77).all()


@pytest.mark.parametrize("n_tgt", [20, 300])
def test_graph_replays_and_two_streams(n_tgt):
    x, c, _ = _inputs(23, 1, 4, 600, n_tgt, 128, "bf16", "mxfp4")
    y, e, _ = _inputs(24, 1, 4, 600, n_tgt, 128, "bf16", "mxfp4")
    run = lambda x, c, **kw: ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], **kw)
    a, b = run(x, c).o_tgt.clone(), run(y, e).o_tgt.clone()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        ra = run(x, c)
    with torch.cuda.stream(t):
        rb = run(y, e)
    torch.cuda.synchronize()
    assert torch.equal(ra.o_tgt, a) and torch.equal(rb.o_tgt, b)
    ws = ops.attn_mx_workspace(x["q_tgt"], 600, "mxfp4")
    out, mass = torch.empty_like(a), torch.empty((1, 4, n_tgt), device="cuda:0")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            run(x, c, o_tgt=out, ref_mass=mass, workspace=ws)
    for rep in range(3):
        src, want = ((y, b), (x, a), (y, b))[rep]
        cache = e if src is y else c
        keep = {n: src[n].clone() for n in ("q_tgt", "k_tgt", "v_tgt")}, cache["k"].codes.clone(), \
            cache["k"].scales.clone(), cache["v"].codes.clone(), cache["v"].scales.clone()
        old = {n: x[n].clone() for n in keep[0]}, c["k"].codes.clone(), c["k"].scales.clone(), \
            c["v"].codes.clone(), c["v"].scales.clone()
        for put in (keep, None, old):
            if put is None:
                torch.cuda.synchronize()
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, want), rep
                continue
            for n, v in put[0].items():
                x[n].copy_(v)
            for dst, v in zip((c["k"].codes, c["k"].scales, c["v"].codes, c["v"].scales), put[1:]):
                dst.copy_(v)


@pytest.mark.parametrize("n_tgt", [5, 300])
def test_infinite_target_keys_and_queries(n_tgt):
    """A target key whose scores are all -inf drops out; an infinite query element makes its row NaN and no other."""
    x, c, vals = _inputs(31, 1, 1, 100, n_tgt, 64, "bf16", "mxfp8")
    x["q_tgt"][0, 0, :, 0] = 1.0
    x["k_tgt"][0, 0, 2, 0] = float("-inf")
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"])
    torch.cuda.synchronize()
    keep = [i for i in range(n_tgt) if i != 2]
    y = dict(x, k_tgt=x["k_tgt"][:, :, keep], v_tgt=x["v_tgt"][:, :, keep])
    _check_rows(r.o_tgt, r.ref_mass, None, host(x["q_tgt"]), vals["k"], vals["v"], y, "bf16")
    x["k_tgt"][0, 0, 2, 0] = 0.0
    x["q_tgt"][0, 0, 1, 3] = float("inf")
    r = ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"])
    torch.cuda.synchronize()
    bad = torch.isnan(r.o_tgt[0, 0]).any(-1)
    assert bad.nonzero().flatten().tolist() == [1] and torch.isnan(r.o_tgt[0, 0, 1]).all()


def test_clock_probe_counts_where_the_cache_is_read_back():
    x, c, _ = _inputs(37, 1, 2, 64, 300, 64, "bf16", "mxfp4")
    probe = torch.zeros(2, dtype=torch.int64, device="cuda:0")
    word = torch.tensor([ops.REUSE], dtype=torch.int32, device="cuda:0")
    ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], q_mx=c["q"], q_ref=x["q_ref"],
                      k_ref=x["k_ref"], v_ref=x["v_ref"], kvsrc="device", decision=word, clock_probe=probe)
    torch.cuda.synchronize()
    assert (probe > 0).all()


def test_wrong_arguments_are_refused():
    x, c, _ = _inputs(29, 1, 2, 64, 8, 64, "bf16", "mxfp4")
    run = lambda **kw: ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], **{**dict(k_mx=c["k"], v_mx=c["v"]), **kw})
    other = ops.mx_tensor((1, 2, 64, 64), "mxfp8", "cuda:0")
    for kw in (dict(kvsrc="fresh"), dict(v_mx=other), dict(v_mx=c["v"].rows(63)), dict(decision=torch.zeros(1)),
               dict(kvsrc="device", decision=torch.zeros(1, device="cuda:0")), dict(ref_mass=torch.zeros(3))):
        with pytest.raises(ValueError):
            run(**kw)
    for kw in (dict(qset="all"), dict(kvsrc="device", q_mx=c["q"]),
               dict(qset="all", q_mx=c["q"], workspace=torch.empty(16, dtype=torch.uint8, device="cuda:0"))):
        with pytest.raises(ops.L.RefadaptError):
            run(**kw)
    torch.cuda.synchronize()
