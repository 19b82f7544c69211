"""Attention over a quantised cache by each of its ways, at sizes that are seen to take it: few target rows with one
key range, few with several ranges and their merge, and the cache read back. Workspaces with guards, poisoned rows
behind the ends, NaN and infinite keys, captured and overlapping calls. Tolerances: those of test_gpu_attn_mx."""

import numpy as np
import pytest
import torch

from gpu_helpers import host
from paper_2609_32415_amd import ops
from test_gpu_attn_mx import _check_rows, _inputs

pytestmark = pytest.mark.gpu

# way: n_ref, n_tgt, heads, bytes of workspace or none
WAYS = {"one range": (333, 33, 3, False), "ranges": (5000, 9, 2, True), "read back": (300, 1100, 2, True)}
FORMATS = ["mxfp4", "mxfp8"]


def _case(way, fmt, d=128, dtype="bf16", seed=3):
    n_ref, n_tgt, H, needs = WAYS[way]
    x, c, vals = _inputs(seed, 1, H, n_ref, n_tgt, d, dtype, fmt)
    assert (ops.attn_mx_workspace(x["q_tgt"], n_ref, fmt).numel() > 0) == needs
    return x, c, vals


def _run(x, c, **kw):
    return ops.joint_attn_mx(x["q_tgt"], x["k_tgt"], x["v_tgt"], k_mx=c["k"], v_mx=c["v"], lse=True, **kw)


def _same(a, b):
    """Bits, NaN equal to NaN."""
    both = ((a.o_tgt, b.o_tgt), (a.ref_mass, b.ref_mass), (a.lse, b.lse))
    plain = lambda t: t.nan_to_num(9.0, 8.0, 7.0)
    return all(torch.equal(torch.isnan(p), torch.isnan(q)) and torch.equal(plain(p), plain(q)) for p, q in both)


def _guarded(need):
    buf = torch.full((need + 8192,), 77, dtype=torch.uint8, device="cuda:0")
    return buf, buf[4096:4096 + need]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", ["ranges", "read back"])
def test_workspace_is_enough_and_not_overrun(way, d, fmt):
    x, c, vals = _case(way, fmt, d)
    need = ops.attn_mx_workspace(x["q_tgt"], c["k"].shape[2], fmt).numel()
    buf, ws = _guarded(need)
    print("workspace", way, d, fmt, need, flush=True)
    r = _run(x, c, workspace=ws)
    torch.cuda.synchronize()
    assert (buf[:4096] == 77).all() and (buf[4096 + need:] == 77).all() and (ws != 77).any()
    _check_rows(r.o_tgt, r.ref_mass, r.lse, host(x["q_tgt"]), vals["k"], vals["v"], x, "bf16")
    with pytest.raises(ops.L.RefadaptError) as e:
        _run(x, c, workspace=ws[:need - 1])
    assert e.value.status == ops.L.RA_EWORKSPACE
    with pytest.raises(ops.L.RefadaptError):
        _run(x, c, workspace=buf[4097:4097 + need])  # not 16-byte aligned


@pytest.mark.parametrize("fmt,dtype,n_ref,n_tgt,qset,kvsrc,cached", [
    ("mxfp4", "bf16", 333, 100, "all", "cache", True), ("mxfp8", "bf16", 2111, 70, "all", "cache", False),
    ("mxfp8", "bf16", 150, 70, "target", "device", True), ("mxfp4", "bf16", 150, 70, "target", "device", False),
    ("mxfp4", "f32", 129, 40, "target", "cache", False), ("mxfp8", "f32", 129, 40, "all", "cache", True)])
def test_read_back_workspaces_of_every_mode(fmt, dtype, n_ref, n_tgt, qset, kvsrc, cached):
    x, c, vals = _inputs(41, 1, 3, n_ref, n_tgt, 64, dtype, fmt)
    need = ops.attn_mx_workspace(x["q_tgt"], n_ref, fmt, qset=qset, kvsrc=kvsrc, q_cached=cached).numel()
    assert need > 0
    buf, ws = _guarded(need)
    kw = dict(qset=qset, kvsrc=kvsrc, q_ref=x["q_ref"], **(dict(q_mx=c["q"]) if cached else {}))
    for dec in (ops.REUSE, ops.REACTIVATE, ops.COMPUTE) if kvsrc == "device" else (None,):
        if dec is not None:
            kw.update(k_ref=x["k_ref"], v_ref=x["v_ref"],
                      decision=torch.tensor([dec], dtype=torch.int32, device="cuda:0"))
        print("read back", fmt, dtype, qset, kvsrc, cached, dec, flush=True)
        r = _run(x, c, workspace=ws, **kw)
        torch.cuda.synchronize()
        assert (buf[:4096] == 77).all() and (buf[4096 + need:] == 77).all()
        kr, vr = (host(x["k_ref"]), host(x["v_ref"])) if dec == ops.COMPUTE else (vals["k"], vals["v"])
        _check_rows(r.o_tgt, r.ref_mass, r.lse, host(x["q_tgt"]), kr, vr, x, dtype)
        if dec != ops.REUSE and (qset == "all" or dec is not None):
            q = vals["q"] if cached and dec != ops.COMPUTE else host(x["q_ref"])
            _check_rows(r.o_ref, None, None, q, kr, vr, x, dtype)


def _poisoned(m, rows):
    """The rows of ``m`` at the head of a longer, wider cache whose other bytes read as NaN (scale 255, e4m3 NaN)."""
    B, H, n, w = m.codes.shape
    codes = torch.full((B, H, n + rows, w + 16), 255, dtype=torch.uint8, device="cuda:0")
    scales = torch.full((B, H, n + rows, m.scales.shape[3] + 4), 255, dtype=torch.uint8, device="cuda:0")
    codes[:, :, :n, :w] = m.codes
    scales[:, :, :n, :m.scales.shape[3]] = m.scales
    return ops.MxTensor(codes[:, :, :n, :w], scales[:, :, :n, :m.scales.shape[3]], m.fmt)


def _poisoned_rows(t, rows, cols=8):
    B, H, n, d = t.shape
    buf = torch.full((B, H, n + rows, d + cols), float("nan"), dtype=t.dtype, device="cuda:0")
    buf[:, :, :n, :d] = t
    return buf[:, :, :n, :d]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_ref,n_tgt", [(1, 1), (9, 31), (31, 9), (33, 33), (65, 1), (95, 41), (288, 63), (300, 250),
                                         (5001, 9), (5031, 33), (257, 1057)])
def test_rows_behind_the_last_are_never_used(fmt, d, n_ref, n_tgt):
    """A ragged tile's missing rows have probability zero, which does not hide a NaN in their V; tiles are loaded up to
    24 tiles past the last (for no rows): the buffers go on for that long."""
    x, c, _ = _inputs(n_ref + n_tgt, 1, 2, n_ref, n_tgt, d, "bf16", fmt)
    print("poisoned", fmt, d, n_ref, n_tgt, flush=True)
    tight = _run(x, c)
    y = {n: _poisoned_rows(x[n], 128) for n in ("q_tgt", "k_tgt", "v_tgt")}
    loose = _run(y, {n: _poisoned(c[n], 1100) for n in "kv"})
    torch.cuda.synchronize()
    assert torch.isfinite(loose.o_tgt).all() and torch.isfinite(loose.ref_mass).all()
    assert torch.equal(tight.o_tgt, loose.o_tgt) and torch.equal(tight.ref_mass, loose.ref_mass) and \
        torch.equal(tight.lse, loose.lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("way", list(WAYS))
def test_nan_blocks_reach_what_sees_them(way, fmt):
    x, c, vals = _case(way, fmt)
    n = c["k"].shape[2]
    clean = _run(x, c)
    # V, in the last range's part of head 1: a block of columns, and nothing of the statistics
    c["v"].scales[0, 1, n - 2, 2] = 255
    r = _run(x, c)
    torch.cuda.synchronize()
    assert torch.isnan(r.o_tgt[0, 1, :, 64:96]).all()
    keep = [i for i in range(128) if not 64 <= i < 96]
    assert torch.equal(r.o_tgt[0, 1][:, keep], clean.o_tgt[0, 1][:, keep])
    assert torch.equal(r.o_tgt[0, 0], clean.o_tgt[0, 0])
    assert torch.equal(r.ref_mass, clean.ref_mass) and torch.equal(r.lse, clean.lse)
    # K, one block in the middle of head 0: every row and statistic of the head, no other
    for row in (0, n // 2, n - 1):
        old = int(c["k"].scales[0, 0, row, 1])
        c["k"].scales[0, 0, row, 1] = 255
        r2 = _run(x, c)
        c["k"].scales[0, 0, row, 1] = old
        torch.cuda.synchronize()
        assert torch.isnan(r2.o_tgt[0, 0]).all() and torch.isnan(r2.ref_mass[0, 0]).all() and \
            torch.isnan(r2.lse[0, 0]).all()
        assert torch.equal(r2.ref_mass[0, 1], clean.ref_mass[0, 1]) and torch.equal(r2.lse[0, 1], clean.lse[0, 1])
        assert torch.equal(r2.o_tgt[0, 1][:, keep], clean.o_tgt[0, 1][:, keep])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("way", list(WAYS))
def test_target_keys_and_values_without_a_number(way, fmt):
    """A NaN target key: every row, its mass and total log-sum-exp, not the reference's. One of -inf scores: as if it
    were not there. A NaN query element: its row alone."""
    x, c, vals = _case(way, fmt)
    n_tgt = x["q_tgt"].shape[2]
    x["q_tgt"][0, 0, :, 0] = 1.0
    clean = _run(x, c)
    old = x["k_tgt"][0, 0, 5, 0].clone()
    x["k_tgt"][0, 0, 5, 0] = float("nan")
    r = _run(x, c)
    torch.cuda.synchronize()
    assert torch.isnan(r.o_tgt[0, 0]).all() and torch.isnan(r.ref_mass[0, 0]).all()
    assert torch.isnan(r.lse[0, 0, :, 1]).all()
    assert torch.isfinite(r.lse[0, 0, :, 0]).all() and torch.equal(r.o_tgt[0, 1], clean.o_tgt[0, 1])
    x["k_tgt"][0, 0, 5, 0] = float("-inf")
    r = _run(x, c)
    torch.cuda.synchronize()
    keep = [i for i in range(n_tgt) if i != 5]
    y = {n: x[n][:, :1] for n in ("q_tgt", "k_tgt", "v_tgt")}
    y = dict(y, k_tgt=y["k_tgt"][:, :, keep], v_tgt=y["v_tgt"][:, :, keep])
    _check_rows(r.o_tgt[:, :1], r.ref_mass[:, :1], r.lse[:, :1], host(y["q_tgt"]), vals["k"][:, :1], vals["v"][:, :1],
                y, "bf16")
    x["k_tgt"][0, 0, 5, 0] = old
    x["q_tgt"][0, 0, 3, 7] = float("nan")
    r = _run(x, c)
    torch.cuda.synchronize()
    assert torch.isnan(r.o_tgt[0, 0, 3]).all() and torch.isnan(r.ref_mass[0, 0, 3])
    # The rows beside it are formed against maxima that its tiles moved, at other roundings: not the same bits.
    rows = [i for i in range(n_tgt) if i != 3]
    y = {n: x[n][:, :1] for n in ("k_tgt", "v_tgt")}
    _check_rows(r.o_tgt[:, :1, rows], r.ref_mass[:, :1, rows], r.lse[:, :1, rows], host(x["q_tgt"])[:, :1, rows],
                vals["k"][:, :1], vals["v"][:, :1], y, "bf16")
    assert torch.equal(r.o_tgt[0, 1], clean.o_tgt[0, 1])


@pytest.mark.parametrize("share", [1.0, 0.5])
@pytest.mark.parametrize("way", list(WAYS))
def test_reference_rows_without_weight(way, share):
    """Reference keys whose scores overflow to -inf (2^100 times -2^100), all of them or the first half: no part of the
    outputs; with none left the mass is 0 and the reference's log-sum-exp -inf."""
    x, c, vals = _case(way, "mxfp8")
    n = c["k"].shape[2]
    k = torch.from_numpy(vals["k"]).to(torch.bfloat16).to("cuda:0")
    k[..., 0] = 0.0
    x["k_tgt"][..., 0] = 0.0
    x["q_tgt"][..., 0] = 2.0 ** 100
    gone = int(n * share)
    k[:, :, :gone, 0] = -2.0 ** 100
    ops.mx_commit(k, None, c["k"], None)
    r = _run(x, c)
    torch.cuda.synchronize()
    kv, = ops.mx_read(c["k"])
    q = host(x["q_tgt"])
    q[..., 0] = 0.0  # the keys that are left have zeros there
    if share == 1.0:
        z = np.zeros((*vals["k"].shape[:2], 0, vals["k"].shape[3]))
        _check_rows(r.o_tgt, r.ref_mass, None, q, z, z, x, "bf16")
        assert (r.ref_mass == 0).all() and torch.isneginf(r.lse[..., 0]).all()
    else:
        _check_rows(r.o_tgt, r.ref_mass, r.lse, q, host(kv)[:, :, gone:], vals["v"][:, :, gone:], x, "bf16")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("way", ["ranges", "read back"])
def test_captured_calls_and_two_streams(way, fmt):
    xs = [_case(way, fmt, seed=s) for s in (51, 52, 53)]
    n_ref = xs[0][1]["k"].shape[2]
    want = [_run(x, c) for x, c, _ in xs]
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(4):  # calls that may overlap, a workspace each
        for stream, (x, c, _) in zip((s, t), xs):
            with torch.cuda.stream(stream):
                got.append(_run(x, c))
    torch.cuda.synchronize()
    assert all(_same(g, want[i % 2]) for i, g in enumerate(got))
    x, c, _ = xs[2]
    ws = ops.attn_mx_workspace(x["q_tgt"], n_ref, fmt)
    assert ws.numel() > 0
    live = {n: x[n].clone() for n in ("q_tgt", "k_tgt", "v_tgt")}
    cache = {n: ops.MxTensor(c[n].codes.clone(), c[n].scales.clone(), fmt) for n in "kv"}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            a = _run(live, cache, workspace=ws)
            b = _run(live, cache, workspace=ws)  # one after the other: one workspace serves both
    for rep in range(6):
        i = rep % 3
        for n, v in live.items():
            v.copy_(xs[i][0][n])
        for n in "kv":
            cache[n].codes.copy_(xs[i][1][n].codes)
            cache[n].scales.copy_(xs[i][1][n].scales)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert _same(a, want[i]) and _same(b, want[i]), rep
        again = _run(xs[i][0], xs[i][1])  # the program's own work between the replays
        torch.cuda.synchronize()
        assert _same(again, want[i])
