"""Layer norm of rows as long as few are: gradients of 2^25 columns and more."""
import pytest
import torch

from paper_1810_09868_amd import binding as B

from gpu_util import TDT, ws_bytes

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5


# around the first that takes all of a launch's 2^32 threads at 16 columns to a workgroup, and the first that meets a workgroup twice
@pytest.mark.parametrize("dtype,N,C", [(B.F32, 1, (1 << 25) + 3), (B.F32, 3, 1 << 25), (B.BF16, 2, (1 << 25) - 5), (B.F32, 2, 1 << 19), (B.F32, 2, (1 << 19) + 9)])
def test_gradients_of_very_long_rows(dtype, N, C):
    gen = torch.Generator(device="cuda").manual_seed(N + C)
    x = (torch.randn((N, C), generator=gen, device="cuda") + 0.25).to(TDT[dtype])
    dy = torch.randn((N, C), generator=gen, device="cuda").to(TDT[dtype])
    gamma = torch.rand((C,), generator=gen, device="cuda") + 0.5
    y, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((N, 2), device="cuda")
    dgamma, dbeta = (torch.full((C + 64,), 3.0, device="cuda") for _ in range(2))
    B.vgg_layer_norm(dtype, N, C, x, gamma, None, EPS, 0.0, None, 0, y, stats)
    ws = ws_bytes(B.vgg_layer_norm_bwd_workspace_bytes(dtype, dtype, N, C))
    B.vgg_layer_norm_bwd(dtype, dtype, N, C, x, gamma, stats, 0.0, None, 0, dy, dx, dgamma, dbeta, False, ws)
    torch.cuda.synchronize()
    assert (dgamma[C:] == 3.0).all() and (dbeta[C:] == 3.0).all()
    half = {B.F32: U, B.BF16: 2.0 ** -8}[dtype]
    # A thread adds up to C / 1024 values, eight at a time, then 12 additions: sums are off by n u of the sum of magnitudes.
    n = C / 8192 + 30
    xd, g = x.double(), dy.double()
    mean = xd.mean(1, keepdim=True)
    X = xd.abs().mean(1, keepdim=True)
    rstd = 1 / ((xd - mean).square().mean(1, keepdim=True) + EPS).sqrt()
    # the mean by n u of X, the width by n / 2 u and what the mean's shift leaves of it; xh by both
    e_mean = n * U * X * rstd
    xh = (xd - mean) * rstd
    e_xh = e_mean + xh.abs() * ((n / 2 + 8) * U + e_mean) + 4 * U * (xd.abs() * rstd)
    assert ((y.double() - xh * gamma).abs() <= gamma * (e_xh + 4 * U * xh.abs()) + half * (xh * gamma).abs()).all()
    gx = g * xh
    assert ((dgamma[:C].double() - gx.sum(0)).abs() <= (g.abs() * e_xh).sum(0) + (N + 4) * U * gx.abs().sum(0)).all()
    assert ((dbeta[:C].double() - g.sum(0)).abs() <= (N + 4) * U * g.abs().sum(0)).all()
    gg = g * gamma
    m1, m2 = gg.mean(1, keepdim=True), (gg * xh).mean(1, keepdim=True)
    dx_want = rstd * (gg - m1 - xh * m2)
    a1, a2 = gg.abs().mean(1, keepdim=True), (gg * xh).abs().mean(1, keepdim=True)
    e2 = (n + 8) * U * a2 + (gg.abs() * e_xh).mean(1, keepdim=True)
    tol = rstd * (4 * U * gg.abs() + (n + 8) * U * a1 + e_xh * m2.abs() + xh.abs() * e2 + 4 * U * (m1.abs() + (xh * m2).abs())) + ((n / 2 + 8) * U + e_mean) * dx_want.abs()
    assert ((dx.double() - dx_want).abs() <= tol + half * dx_want.abs()).all()
