"""Offsets past 32 bits: rows and heads of the operators' tensors gigabytes apart, against the same values held close."""

import pytest
import torch

from paper_2609_32415_amd import ops

pytestmark = pytest.mark.gpu

GB = 1 << 30


def _far(x, stride_h, stride_s, pool):
    """The values of x [1, H, n, d] at these strides (elements) in a large buffer of bytes."""
    buf = pool.view(x.dtype) if x.dtype != torch.uint8 else pool
    y = buf.as_strided(x.shape, (0, stride_h, stride_s, 1))
    y.copy_(x)
    return y


@pytest.fixture(scope="module")
def pool():
    # rows 2^24 - 16 elements apart: 300 rows of bf16 span 10 GB, of bytes 5 GB
    p = torch.empty(11 * GB, dtype=torch.uint8, device="cuda:0")
    yield p
    del p
    torch.cuda.empty_cache()


ROW, N = (1 << 24) - 16, 300


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_cache_rows_far_apart(fmt, pool):
    x = torch.randn((1, 1, N, 64), device="cuda:0").to(torch.bfloat16)
    near = ops.mx_tensor(x.shape, fmt, "cuda:0")
    ops.mx_commit(x, None, near, None)
    print("far rows: commit", fmt, flush=True)
    far_x = _far(x, 0, ROW, pool)
    m = ops.mx_tensor(x.shape, fmt, "cuda:0")
    ops.mx_commit(far_x, None, m, None)
    torch.cuda.synchronize()
    assert torch.equal(m.codes, near.codes) and torch.equal(m.scales, near.scales)
    far_x.fill_(0)
    print("far rows: read", fmt, flush=True)
    ops.mx_read(near, k_out=far_x)
    torch.cuda.synchronize()
    assert torch.equal(far_x, ops.mx_read(near)[0])
    # a cache with far rows, attended over straight and read back
    far = ops.MxTensor(_far(near.codes, 0, ROW, pool), near.scales, fmt)
    for n_tgt in (7, 1100):
        q, k, v = (torch.randn((1, 1, n_tgt, 64), device="cuda:0").to(torch.bfloat16) for _ in range(3))
        print("far rows: attention", fmt, n_tgt, flush=True)
        a = ops.joint_attn_mx(q, k, v, k_mx=near, v_mx=near)
        b = ops.joint_attn_mx(q, k, v, k_mx=far, v_mx=far)
        torch.cuda.synchronize()
        assert torch.equal(a.o_tgt, b.o_tgt) and torch.equal(a.ref_mass, b.ref_mass)


def test_heads_far_apart(pool):
    stride = 5 * GB // 2  # elements of bf16
    x = torch.randn((1, 2, 40, 64), device="cuda:0").to(torch.bfloat16)
    far = _far(x, stride, 64, pool)
    freq, axis = ops.rope_frequencies((32, 32))
    pos = torch.randint(0, 99, (40, 2), dtype=torch.int32, device="cuda:0")
    print("far heads", flush=True)
    want = ops.rope(x, pos=pos, freq=freq, axis=axis)
    near, m = (ops.mx_tensor(x.shape, "mxfp8", "cuda:0") for _ in range(2))
    ops.mx_commit(x, None, near, None)
    ops.mx_commit(far, None, m, None)
    got = ops.rope(far, pos=pos, freq=freq, axis=axis, q_out=far)
    torch.cuda.synchronize()
    assert torch.equal(m.codes, near.codes) and torch.equal(got, want)
    far = _far(x, stride, 64, pool)
    assert torch.equal(ops.rope(far, pos=pos, freq=freq, axis=axis, pairing="half", q_out=far),
                       ops.rope(x, pos=pos, freq=freq, axis=axis, pairing="half"))
    codes = pool.as_strided(near.codes.shape, (0, 5 * GB, 64, 1))
    codes.copy_(near.codes)
    q, k, v = (torch.randn((1, 2, 9, 64), device="cuda:0").to(torch.bfloat16) for _ in range(3))
    f = ops.MxTensor(codes, near.scales, "mxfp8")
    a = ops.joint_attn_mx(q, k, v, k_mx=near, v_mx=near)
    b = ops.joint_attn_mx(q, k, v, k_mx=f, v_mx=f)
    torch.cuda.synchronize()
    assert torch.equal(a.o_tgt, b.o_tgt)
