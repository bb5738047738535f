"""Layer norm and its gradient in place, of more rows than run at once: the same bits as apart."""
import pytest
import torch

from paper_1810_09868_amd import binding as B

from gpu_util import ws_bytes
from test_gpu_norm import EPS, Norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("N,C", [(9000, 5), (40000, 40), (5000, 700), (3000, 4099), (700, 9000), (600, 20000), (600, 28672), (1100, 30001)])
def test_in_place_as_apart(dtype, N, C):
    n = Norm(dtype, N, C, 13, relu=True)
    n.forward().backward()
    y, dx, x = n.y.clone(), n.dx.clone(), n.xs.clone()
    n.forward(y=n.xs)
    assert torch.equal(n.xs, y)
    n.xs.copy_(x)
    n.backward(in_place=True)
    assert torch.equal(n.dx, dx)
    dy = n.dy.cuda()
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = ws_bytes(B.vgg_layer_norm_bwd_workspace_bytes(dtype, dtype, N, C))
    B.vgg_layer_norm_bwd(dtype, dtype, N, C, n.xs, n.gd, n.stats, 0.0, None, n.layer, dy, n.xs, dgamma, dbeta, True, ws)
    assert torch.equal(n.xs, dx) and torch.equal(dgamma, n.dgamma) and torch.equal(dbeta, n.dbeta)
