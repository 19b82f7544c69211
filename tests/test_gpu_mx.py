"""The quantised reference cache against the fp64 oracle: codes, scales and values have one right answer each, so
everything is compared for equality."""

import numpy as np
import pytest
import torch

from gpu_helpers import TORCH_DTYPE
from oracle import mx as oracle_mx
from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu

FORMATS = ("mxfp4", "mxfp8")


def _same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def _check(m, x):
    """An MxTensor against the oracle's codes and scales of the plain tensor, and its values read back."""
    xs = x.double().cpu().numpy()
    code, scale = oracle_mx.quantise(xs, m.fmt)
    codes = oracle_mx.pack(code, m.fmt)
    assert _same(m.scales.cpu().numpy(), scale)
    assert _same(m.codes.cpu().numpy(), codes)
    want = oracle_mx.values(codes, scale, m.fmt)
    for dtype in (torch.bfloat16, torch.float32):
        v, = ops.mx_read(m, dtype=dtype)
        assert v.dtype == dtype and _same(v.double().cpu().numpy(), want)


def _values(rng, shape, dtype, wide):
    x = rng.standard_normal(shape)
    if wide:  # every exponent of the type, signed zeros and blocks of zeros
        x = np.ldexp(x, rng.integers(-140, 127, shape))
        x *= rng.random(shape) > 0.1
        x[..., :1, :32] = -0.0
    return torch.from_numpy(x.astype(np.float32)).to(TORCH_DTYPE[dtype]).to("cuda:0")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,n,d,wide", [(1, 1, 1, 32, False), (1, 2, 7, 64, True), (2, 3, 130, 128, False),
                                          (1, 5, 77, 96, True), (2, 1, 1025, 128, True), (1, 24, 65, 64, False)])
def test_commit_and_read(fmt, dtype, B, H, n, d, wide):
    rng = np.random.default_rng(n + d)
    k, v, q = (_values(rng, (B, H, n, d), dtype, wide) for _ in range(3))
    v = v.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # heads beside the channels
    mk, mv, mq = (ops.mx_tensor(k.shape, fmt, "cuda:0") for _ in range(3))
    print("mx", fmt, dtype, B, H, n, d, flush=True)
    ops.mx_commit(k, v, mk, mv, q_ref=q, q_mx=mq)
    torch.cuda.synchronize()
    for m, x in ((mk, k), (mv, v), (mq, q)):
        _check(m, x)
    got = ops.mx_read(mk, mv, mq, dtype=TORCH_DTYPE[dtype])
    alone = [ops.mx_read(m, dtype=TORCH_DTYPE[dtype])[0] for m in (mk, mv, mq)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, alone))


@pytest.mark.parametrize("fmt", FORMATS)
def test_borders_ties_and_largest_values(fmt):
    """Blocks whose largest magnitude lies at, just below and just above the border of two scales, at every exponent of
    bf16; values on the midpoints between codes; the largest and smallest finite values."""
    top, emax = (7.0, 2) if fmt == "mxfp4" else (464.0, 8)
    rows = []
    mids = np.convolve(oracle_mx.FORMATS[fmt][0], [0.5, 0.5], "valid")
    for e in range(-133, 128 - emax):
        for a in (top, np.nextafter(np.float32(top), np.float32(0)), np.nextafter(np.float32(top), np.float32(1e9))):
            r = np.resize(mids, 32) * np.resize([1, -1, 1], 32)
            r[e % 32] = a
            rows.append(np.ldexp(r, e))
    rows.append(np.resize([3.4028235e38, -3.3895e38, 1e-45, -1e-38], 32))
    x = torch.from_numpy(np.clip(np.array(rows), -3.4028235e38, 3.4028235e38).astype(np.float32))
    for dtype in (torch.float32, torch.bfloat16):
        y = x.to(dtype).nan_to_num(posinf=3.3895e38, neginf=-3.3895e38).view(1, 1, -1, 32).to("cuda:0")
        m = ops.mx_tensor(y.shape, fmt, "cuda:0")
        ops.mx_commit(y, None, m, None)
        torch.cuda.synchronize()
        _check(m, y)


@pytest.mark.parametrize("fmt", FORMATS)
def test_nan_and_infinity_stay_in_their_block(fmt):
    x = torch.ones((1, 1, 4, 64), dtype=torch.bfloat16, device="cuda:0")
    x[0, 0, 0, 3], x[0, 0, 1, 40], x[0, 0, 2, 63] = float("nan"), float("inf"), float("-inf")
    m = ops.mx_tensor(x.shape, fmt, "cuda:0")
    ops.mx_commit(x, None, m, None)
    torch.cuda.synchronize()
    _check(m, x)
    bad = torch.isnan(ops.mx_read(m)[0]).cpu()
    assert bad.view(4, 2, 32).all(-1).tolist() == [[True, False], [False, True], [False, True], [False, False]]


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_code_under_every_scale_reads_exactly(fmt):
    d = 32
    codes = np.arange(256, dtype=np.uint8).reshape(-1, d if fmt == "mxfp8" else d // 2)
    rows = codes.shape[0]
    m = ops.mx_tensor((1, 1, 256 * rows, d), fmt, "cuda:0")
    m.codes.copy_(torch.from_numpy(np.tile(codes, (256, 1))))
    m.scales.copy_(torch.from_numpy(np.repeat(np.arange(256), rows).astype(np.uint8))[:, None])
    want = oracle_mx.values(np.tile(codes, (256, 1)), np.repeat(np.arange(256), rows).astype(np.uint8)[:, None], fmt)
    got = torch.from_numpy(want).to(torch.bfloat16).double().numpy()  # scales below the lowest round, those above overflow
    out, = ops.mx_read(m)
    torch.cuda.synchronize()
    lo, hi = (0, 252) if fmt == "mxfp4" else (3, 246)
    keep = np.repeat((np.arange(256) >= lo) & (np.arange(256) <= hi) | (np.arange(256) == 255), rows)
    assert _same(out[0, 0].double().cpu().numpy()[keep], want[keep])
    assert _same(got[keep], want[keep])


@pytest.mark.parametrize("fmt", FORMATS)
def test_decision_age_and_rows_behind_the_last(fmt):
    """Only COMPUTE writes; a cache for more rows keeps those behind n_ref, and codes and scales with padded rows."""
    rng = np.random.default_rng(1)
    B, H, n, d = 1, 3, 21, 64
    k = _values(rng, (B, H, n, d), "bf16", False)
    big = ops.mx_tensor((B, H, n + 4, 2 * d), fmt, "cuda:0")
    m = ops.MxTensor(big.codes[..., :big.codes.shape[3] // 2], big.scales[..., :2], fmt).rows(n)
    age = torch.full((1,), 7, dtype=torch.int32, device="cuda:0")
    for dec in (ops.REUSE, ops.REACTIVATE, ops.COMPUTE):
        big.codes.fill_(171)
        big.scales.fill_(99)
        word = torch.tensor([dec], dtype=torch.int32, device="cuda:0")
        ops.mx_commit(k, None, m, None, decision=word, age=age, step=5)
        torch.cuda.synchronize()
        if dec == ops.COMPUTE:
            assert age.item() == 5
            _check(m, k)
            m.codes.fill_(171)
            m.scales.fill_(99)
        else:
            assert age.item() == 7
        assert (big.codes == 171).all() and (big.scales == 99).all()


def test_graph_replays_follow_the_decision():
    x = torch.randn((1, 2, 50, 64), device="cuda:0").to(torch.bfloat16)
    m = ops.mx_tensor(x.shape, "mxfp4", "cuda:0")
    out = torch.empty_like(x)
    dec = torch.tensor([ops.COMPUTE], dtype=torch.int32, device="cuda:0")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()

    def call():
        ops.mx_commit(x, None, m, None, decision=dec)
        ops.mx_read(m, k_out=out)

    with torch.cuda.stream(s):
        call()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            call()
    kept = None
    for d in (ops.COMPUTE, ops.REUSE, ops.COMPUTE, ops.REACTIVATE):
        x.copy_(torch.randn(x.shape, device="cuda:0"))
        dec.fill_(d)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        if d == ops.COMPUTE:
            e = ops.mx_tensor(x.shape, "mxfp4", "cuda:0")
            ops.mx_commit(x, None, e, None)
            kept, = ops.mx_read(e)
        assert torch.equal(out, kept)


def test_wrong_tensors_are_refused():
    x = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16, device="cuda:0")
    m = ops.mx_tensor(x.shape, "mxfp4", "cuda:0")
    m8 = ops.mx_tensor(x.shape, "mxfp8", "cuda:0")
    for call in (lambda: ops.mx_commit(x, x, m, None), lambda: ops.mx_commit(x, x, m, m8),
                 lambda: ops.mx_commit(x[:, :, :7], None, m, None), lambda: ops.mx_commit(x, None, m, None, q_ref=x),
                 lambda: ops.mx_commit(x.half(), None, m, None), lambda: ops.mx_commit(x.cpu(), None, m, None),
                 lambda: ops.mx_commit(x, None, ops.MxTensor(m.codes, m.scales[..., :1], "mxfp4"), None),
                 lambda: ops.mx_commit(x, None, ops.MxTensor(m.codes.int(), m.scales, "mxfp4"), None),
                 lambda: ops.mx_commit(x, None, m, None, decision=torch.zeros(1, device="cuda:0")),
                 lambda: ops.mx_read(m, v_out=x), lambda: ops.mx_read(m, k_out=x.float()),
                 lambda: ops.mx_read(m, dtype=torch.float16), lambda: ops.mx_tensor((1, 1, 1, 48), "mxfp4", "cuda:0"),
                 lambda: ops.mx_tensor((1, 1, 1, 64), "fp4", "cuda:0")):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
