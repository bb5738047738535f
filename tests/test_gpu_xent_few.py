"""Losses of few fp32 rows over many classes, whose scores and their gradients come from weights where they are: masks that leave nothing, rows that do
not count, NaN, masked classes' weights, parts of the gradient, another stream, a graph."""
import math

import pytest
import torch

from paper_1810_09868_amd import binding as B

from gpu_util import ws_bytes
from test_gpu_xent import Xent

pytestmark = pytest.mark.gpu

SIZES = [(1, 64, 16384), (7, 129, 16641), (32, 70, 20000), (33, 256, 16385), (64, 40, 20003), (3, 4096, 40000)]
GRADIENTS = ("da", "dw", "db")


def held(c):
    return {k: getattr(c, k).clone() for k in ("loss",) + GRADIENTS}


@pytest.mark.parametrize("N,In,K", SIZES)
def test_masks_and_rows_that_do_not_count(N, In, K):
    c = Xent(B.F32, N, In, K, 31, masked=0.4)
    c.labels[0] = int(torch.nonzero(c.bias == -math.inf)[0])             # a masked label
    c.run().check()
    assert c.loss[0] == math.inf
    want = held(c)
    c.w[c.bias == -math.inf] = 1e30                                      # weights of masked classes
    c.run()
    assert all(torch.equal(getattr(c, k), v) for k, v in want.items())
    c = Xent(B.F32, N, In, K, 32)
    c.labels[torch.arange(N) % 3 == 0] = -1
    if N > 4:
        c.labels[1], c.labels[4] = 2 ** 31 - 1, -2 ** 31
        c.labels[5], c.g[5] = 2, 0
    out = ~((c.labels >= 0) & (c.labels < K))
    c.run().check()
    want = held(c)
    for bad in (math.nan, math.inf):
        c.a[out] = bad
        if N > 4:
            c.a[5] = bad
        c.run()
        assert torch.equal(c.dw, want["dw"]) and torch.equal(c.db, want["db"]) and (c.da[out] == 0).all() and (c.loss[out] == 0).all()
    c = Xent(B.F32, N, In, K, 33)
    c.bias[:] = -math.inf                                                # nothing is left
    c.run().check()
    assert (c.stats == -math.inf).all() and (c.da == 0).all() and (c.dw == 0).all() and (c.db == 0).all()
    c.bias[K - 1] = 0.5                                                  # one class is
    c.labels[:] = K - 1
    c.run().check()
    assert (c.loss == 0).all() and (c.da == 0).all() and (c.dw == 0).all()


@pytest.mark.parametrize("N,In,K", SIZES[1:])
def test_nan_and_infinite_scores(N, In, K):
    c = Xent(B.F32, N, In, K, 34)
    c.labels[:] = 7
    c.run()
    want = held(c)
    c.a[2, 5] = math.nan
    c.run()
    rest = torch.arange(N, device="cuda") != 2
    assert torch.isnan(c.loss[2]) and torch.equal(c.loss[rest], want["loss"][rest]) and torch.equal(c.da[rest], want["da"][rest])
    assert c.g[2] == 0 or (torch.isnan(c.da[2]).all() and torch.isnan(c.db).all())
    c.a[2, 5] = 1.0
    c.bias[9] = math.inf
    c.run()
    assert torch.isnan(c.loss).all()


@pytest.mark.parametrize("N,In,K", SIZES)
def test_parts_of_the_gradient_other_streams_and_a_graph(N, In, K):
    c = Xent(B.F32, N, In, K, 35, masked=0.1)
    c.a.clamp_min_(0)
    c.run()
    want = held(c)
    for part in (("da",), ("dw",), ("db",), ("dw", "db")):
        c.run(part)
        assert all(torch.equal(getattr(c, k), want[k]) for k in part)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(getattr(c, k), v) for k, v in want.items())
    ws = ws_bytes(max(B.vgg_fc_xent_workspace_bytes(B.F32, N, In, K), B.vgg_fc_xent_bwd_workspace_bytes(B.F32, N, In, K)))
    da = torch.empty_like(c.da)
    B.vgg_fc_xent_bwd(B.F32, B.F32, N, In, K, c.a, c.w, c.bias, c.labels, c.stats, c.g, da, None, None, ws, relu_mask=True)
    assert torch.equal(da, torch.where(c.a > 0, want["da"], 0.0))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.vgg_fc_xent(B.F32, N, In, K, c.a, c.w, c.bias, c.labels, c.loss, c.stats, ws)
        B.vgg_fc_xent_bwd(B.F32, B.F32, N, In, K, c.a, c.w, c.bias, c.labels, c.stats, c.g, c.da, c.dw, c.db, ws)
    for seed in (36, 37, 38):
        other = Xent(B.F32, N, In, K, seed).run()
        for k in ("a", "w", "bias", "labels", "g"):
            getattr(c, k).copy_(getattr(other, k))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(c, k), v) for k, v in held(other).items())
