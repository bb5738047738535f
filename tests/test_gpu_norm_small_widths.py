"""Layer norm of rows that hardly vary: widths whose squares fp32 holds as subnormal numbers only, with eps 0."""
import pytest
import torch

from paper_1810_09868_amd import binding as B

from gpu_util import ws_bytes

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -149


# a team of every kind, and rows longer than a workgroup holds
@pytest.mark.parametrize("C", [2, 7, 64, 333, 700, 4096, 9000, 20000, 40000])
@pytest.mark.parametrize("power", [-50, -64, -66, -70])
def test_variances_that_are_subnormal(C, power):
    # Values of -1, 0 and 1 times a power of two, as many of either sign: the mean is 0, and as it is computed, from means of waves, 48 u of the largest value at
    # the most.  Squares of subnormal size are rounded to whole 2^-149, half a step for each of the C and for the few that join waves, which leaves up to
    # (C + 16) / 2 steps in their sum, one and 8 / C in the variance after its own rounding, and half of that, relative, in rstd; beside it the 60 u of rows of ordinary size.
    N = 3
    gen = torch.Generator(device="cuda").manual_seed(C)
    half = torch.rand((N, C // 2), generator=gen, device="cuda") < 0.8
    half[:, 0] = True
    x = torch.zeros((N, C), device="cuda")
    x[:, :C // 2], x[:, C - C // 2:] = half.float(), -half.float()
    x *= 2.0 ** power
    y, stats = torch.empty_like(x), torch.empty((N, 2), device="cuda")
    B.vgg_layer_norm(B.F32, N, C, x, None, None, 0.0, 0.0, None, 0, y, stats)
    xd = x.double()
    var = xd.square().mean(1, keepdim=True)
    off = 0.5 * (1 + 8 / C) * TINY / var + 60 * U
    assert float(off.max()) < 0.01 and (stats[:, 0].abs() <= 48 * U * 2.0 ** power).all()
    assert ((stats[:, 1:].double() * var.sqrt() - 1).abs() <= off).all()
    assert ((y.double() * var.sqrt() - xd).abs() <= xd.abs() * (off + 2 * U) + 50 * U * 2.0 ** power).all()
    # and the gradient takes the same rstd
    dy = torch.randn((N, C), generator=gen, device="cuda") * 2.0 ** power
    dx, dbeta = torch.empty_like(x), torch.empty(C, device="cuda")
    ws = ws_bytes(B.vgg_layer_norm_bwd_workspace_bytes(B.F32, B.F32, N, C))
    B.vgg_layer_norm_bwd(B.F32, B.F32, N, C, x, None, stats, 0.0, None, 0, dy, dx, None, dbeta, False, ws)
    assert torch.isfinite(dx).all() and float(dx.abs().max()) > 0
