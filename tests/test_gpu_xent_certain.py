"""Losses over many classes where labels are all but certain and the scores are products that round: the gradients of such rows hang on the
loss and its gradients taking the same scores, which every path of the kernels has to do."""
import math

import pytest
import torch

from paper_1810_09868_amd import binding as B

from test_gpu_xent import U, Xent

pytestmark = pytest.mark.gpu

# 1 - p of a label is some K exp(-gap): from 1e-3 to 1e-12
BEYOND = (7.0, 11.0, 14.0, 18.0, 21.0, 28.0)
# by the plans: short fp32 products, a split contraction, tiles (fp32: of other columns for the scores than for their gradients), classes in
# pieces, and fp32 weights from where they are: around 32 rows, all of 64, a last tile of one class, pieces, inputs that fill no run
F32 = [(8, 64, 40), (64, 1024, 1000), (100, 4096, 1000), (128, 192, 40000), (257, 256, 30000), (8200, 64, 17000), (4, 1024, 10007), (65, 64, 20000),
       (1, 512, 16384), (8, 1024, 40000), (8, 256, 16641), (31, 129, 20000), (32, 256, 20000), (33, 257, 20001), (64, 512, 16400), (5, 4096, 40000), (7, 3, 30000)]
BF16 = [(8, 64, 40), (100, 4096, 1000), (128, 192, 40000), (257, 256, 30000), (1000, 33, 3000), (8, 1024, 40000)]


def certain(dtype, N, In, K, seed):
    """Every row's label is a class of its own, whose weights point along the row."""
    c = Xent(dtype, N, In, K, seed, std=0.5)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    gap = torch.tensor(BEYOND, device="cuda")[torch.arange(N, device="cuda") % len(BEYOND)] + math.log(K)
    labels = torch.randperm(K, generator=gen, device="cuda")[:N]
    a = c.a.float()
    c.w[labels] = (a * (gap / a.square().sum(1))[:, None]).to(c.w.dtype)
    c.labels = labels.to(torch.int32)
    c.bias.mul_(0.1)
    c.g = 0.5 + torch.rand(N, generator=gen, device="cuda")
    return c


@pytest.mark.parametrize("dtype,N,In,K", [(B.F32, *s) for s in F32] + [(B.BF16, *s) for s in BF16])
def test_gradients_of_labels_that_are_all_but_certain(dtype, N, In, K):
    """As Xent.reference, but a label's dz is held to a part of itself, however small: g (p - 1) is the sum of the others' shares, each exp of a difference of
    two scores, which are off by e_row each.  Beyond that: exponentials, log1p and expm1 of 4 u each, the sum of the shares 100 u; fp32's floor of 2^-39 g
    does not enter db."""
    c = certain(dtype, N, In, K, N + In + K).run()
    a, w = c.a.double(), c.w.double()
    z = a @ w.t() + c.bias.double()
    size = a.abs() @ w.abs().t()
    e_row = ((2 * (In / 16 + 1) * 2 * U + 4 * U) * size + 2 * U * c.bias.double().abs()).amax(1, keepdim=True)
    at = c.labels.long()[:, None]
    share = (z - torch.logsumexp(z, 1, keepdim=True)).exp()
    others = share.scatter(1, at, 0.0)
    missing = others.sum(1, keepdim=True)
    g = c.g.double()[:, None]
    dz = g * others.scatter(1, at, -missing)
    off = dz.abs() * (torch.expm1(2 * e_row) + 120 * U)
    assert float(missing.min()) < 1e-6 or N < len(BEYOND)
    want, tol = dz.sum(0), (off + (N / 32 + 80) * U * dz.abs()).sum(0)
    over = (c.db.double() - want).abs() - tol
    assert float(over.max()) <= 0, float((over / tol).max())
    # the sign, wherever other rows have next to no part in the label's class
    label, alone = c.labels.long(), dz.gather(1, at)[:, 0]
    own = (want[label] / alone - 1).abs() < 0.5
    assert (c.db[label[own]] < 0).all()
    # (each form where it loses nothing: a row of few inputs may score another row's label higher than its own)
    loss = torch.where(missing < 0.5, torch.log1p(missing / (1 - missing)), torch.logsumexp(z, 1, keepdim=True) - z.gather(1, at))[:, 0]
    assert ((c.loss.double() - loss).abs() <= loss * (torch.expm1(2 * e_row[:, 0]) + 120 * U)).all()
    half, floor = (2.0 ** -8, 0.0) if dtype == B.BF16 else (4 * U, 2.0 ** -39)
    want = dz @ w
    tol = (dz.abs() * half + off + floor * g + 4 * (K / 16 + 70) * U * dz.abs()) @ w.abs() + (2.0 ** -8 if dtype == B.BF16 else U) * want.abs()
    assert bool(((c.da.double() - want).abs() <= tol).all())
    want = dz.t() @ a
    tol = (dz.abs() * half + off + floor * g + 4 * (N / 16 + 70) * U * dz.abs()).t() @ a.abs() + (2.0 ** -8 if dtype == B.BF16 else U) * want.abs()
    assert bool(((c.dw.double() - want).abs() <= tol).all())
