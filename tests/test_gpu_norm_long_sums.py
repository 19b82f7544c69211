"""The layer norm's parameter gradients over many rows of many batch entries: their error does not grow with the rows.

Every row is the same, with mean 0 and deviation 1 given as its statistics, so that h is x itself. The sums run in fp32
over chunks of 512 rows at most, which leaves a rounding a row and one of the product, and in fp64 from there on, with
one rounding of the result: 514 of 2^-24 of the sum of the terms' sizes. Up to 1024 columns four wavefronts share a
chunk's rows, and their sums take three more: 133. (Sums of equal terms: in one chunk of 16384 rows they would be off by
up to 2700, and by up to 170 of 1024.)"""

import pytest
import torch

from paper_2609_32415_amd import ops
from test_gpu_norm import U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,S,C", [(512, 16384, 1032), (600, 4097, 24), (3, 70001, 2056), (1, 131072, 4104)])
def test_sums(B, S, C):
    v = 1.0 + torch.arange(C, dtype=torch.float64) % 97 / 100 + 0.003
    row = lambda t: t.to(torch.float32).to("cuda:0")
    dy, x = row(v), row(3.0 - v)
    stats = torch.tensor([0.0, 1.0], device="cuda:0").expand(B, S, 2).contiguous()
    spread = lambda t: t.expand(S, C).contiguous().expand(B, S, C)  # the entries share their rows
    print("long sums", B, S, C, flush=True)
    got = ops.layer_norm_grad(spread(dy), spread(x), stats, wanted=(False, True, True, True, True))[1:]
    P, D = (dy.double() * x.double()) * S, dy.double() * S
    for t, exact in zip(got, (P * B, D * B, P.expand(B, C), D.expand(B, C))):
        assert float(((t.double() - exact).abs() / exact).max()) <= (133 if C <= 1024 else 514) * U
