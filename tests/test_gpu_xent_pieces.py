"""Losses over more classes than a piece holds of few bf16 rows, which keep what rounding leaves of their dz."""
import pytest
import torch

from paper_1810_09868_amd import binding as B

from test_gpu_xent import Xent

pytestmark = pytest.mark.gpu


# by the plans: two pieces each (whole stages of inputs, and weights laid out)
@pytest.mark.parametrize("N,In,K", [(512, 64, 300001), (449, 33, 270000)])
def test_few_bf16_rows_in_pieces(N, In, K):
    c = Xent(B.BF16, N, In, K, 23, masked=0.1)
    c.labels[0], c.labels[1], c.labels[2] = K - 1, 0, 262144          # in the first and the last piece
    c.run().check()
    whole = {k: getattr(c, k).clone() for k in ("da", "dw", "db")}
    c.run()
    assert all(torch.equal(getattr(c, k), v) for k, v in whole.items())
