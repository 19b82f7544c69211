"""The gradient of a projection's bias over many rows: its error does not grow with them.

Every row is the same. A thread adds up 128 rows at most in fp32, three such sums join a fourth, and fp64 takes over,
with one rounding of the result: 132 of 2^-24. (In chunks of 16384 rows it would be off by up to 690.)"""

import numpy as np
import pytest
import torch

from paper_2609_32415_amd import ops
from test_gpu_mx_linear import U, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,S,N", [(1024, 16384, 40), (10, 16384, 24576), (3, 70001, 513)])
def test_bias(B, S, N):
    v = (1.0 + torch.arange(N, dtype=torch.float64) % 97 / 100 + 0.003).to(torch.float32).to("cuda:0")
    w, _ = _weights(np.random.default_rng(0), N, 32, "mxfp4")
    print("long sums", B, S, N, flush=True)
    _, db = ops.mx_linear_grad(v.expand(S, N).contiguous().expand(B, S, N), w, wanted=(False, True))
    exact = v.double() * (B * S)
    assert float(((db.double() - exact).abs() / exact).max()) <= 132 * U
