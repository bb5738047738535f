"""Layer norm, its gradient and dropout against the definitions in 64 bits: one column to rows longer than a workgroup holds, rows of every
alignment, constant rows, NaN, in place, another stream, recorded graphs."""
import numpy as np
import pytest
import torch

from paper_1810_09868_amd import binding as B

from gpu_util import TDT, ws_bytes

pytestmark = pytest.mark.gpu

EPS = 1e-5
HALF = {B.F32: 2.0 ** -24, B.BF16: 2.0 ** -8}      # a rounding's most, relative
U = 2.0 ** -24


def philox(counter, key):
    """Philox 4x32-10 of uint64 arrays that hold 32-bit words."""
    low = np.uint64(0xFFFFFFFF)
    x, k = [np.asarray(c, np.uint64) for c in counter], [np.uint64(v) for v in key]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ x[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return x


def kept(N, C, p, seed, step, layer, rows=None):
    rows = np.arange(N) if rows is None else np.asarray(rows)
    groups = -(-C // 8)
    shape = (len(rows), groups)
    full = lambda v: np.full(shape, v, np.uint64)  # noqa: E731
    seed, step = seed % (1 << 64), step % (1 << 64)
    words = philox((np.broadcast_to(np.arange(groups, dtype=np.uint64), shape), np.broadcast_to(rows.astype(np.uint64)[:, None], shape),
                    full(step & 0xFFFFFFFF), full((step >> 32 & 0xFFFF) | layer << 16)), (seed & 0xFFFFFFFF, seed >> 32))
    numbers = np.stack([w >> np.uint64(s) & np.uint64(0xFFFF) for w in words for s in (0, 16)], -1).reshape(len(rows), -1)[:, :C]
    return numbers >= np.uint64(bar(p))


def bar(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def scale(p):
    return 65536 / (65536 - bar(p)) if bar(p) < 65536 else 0.0


def state(seed, step):
    return torch.tensor([seed - (1 << 64) if seed >= 1 << 63 else seed, step], dtype=torch.int64, device="cuda")


def padded(values, ld, dtype, fill=7e4):
    N, C = values.shape
    buf = torch.full((N, ld), fill, dtype=TDT[dtype])
    buf[:, :C] = torch.as_tensor(values)
    return buf.cuda()


def test_the_generator_itself():
    # the known answers that its authors publish
    assert [int(v) for v in philox([0, 0, 0, 0], [0, 0])] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ff = 0xFFFFFFFF
    assert [int(v) for v in philox([ff] * 4, [ff] * 2)] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("N,C,ldx,ldy,p", [(1, 1, 1, 1, 0.5), (1, 8, 8, 8, 0.1), (3, 7, 7, 9, 0.25), (100, 4096, 4096, 4096, 0.5), (5, 4099, 4103, 4099, 0.1),
                                           (1000, 33, 33, 40, 0.75), (1, 100003, 100003, 100003, 0.5), (7, 64, 72, 65, 1.0), (7, 64, 64, 64, 0.0), (4, 50, 50, 50, 1e-6)])
def test_dropout(dtype, N, C, ldx, ldy, p):
    rng = np.random.default_rng(N * C)
    x = torch.from_numpy(rng.standard_normal((N, C)).astype(np.float32)).to(TDT[dtype])
    seed, step, layer = 0xFEDCBA9876543210, (5 << 33) + 12345, 65535
    xs, y = padded(x, ldx, dtype), torch.full((N, ldy), 3.0, dtype=TDT[dtype], device="cuda")
    B.vgg_dropout(dtype, N, C, xs, p, state(seed, step), layer, y, ldx=ldx, ldy=ldy)
    keep = torch.from_numpy(kept(N, C, p, seed, step, layer))
    want = torch.where(keep, x.float() * np.float32(scale(p)) if bar(p) else x.float(), torch.zeros(())).to(TDT[dtype])
    assert torch.equal(y[:, :C].cpu(), want)
    assert (y[:, C:] == 3.0).all()
    if N * C > 10000 and 0 < p < 1:       # 6 sigma
        assert abs(keep.float().mean().item() - (1 - p)) < 6 * (p * (1 - p) / (N * C)) ** 0.5 + 2 ** -17
    if ldx == ldy:                        # in place
        B.vgg_dropout(dtype, N, C, xs, p, state(seed, step), layer, xs, ldx=ldx, ldy=ldx)
        assert torch.equal(xs[:, :C].cpu(), want)


def test_dropout_of_nan_and_infinity_and_other_seeds_steps_and_layers():
    N, C, p = 4, 1000, 0.5
    x = torch.full((N, C), float("nan"), device="cuda")
    x[:, ::2] = float("inf")
    y = torch.empty_like(x)
    masks = []
    for seed, step, layer in ((1, 0, 0), (2, 0, 0), (1 + (1 << 32), 0, 0), (1, 1, 0), (1, 1 << 32, 0), (1, 0, 1)):
        B.vgg_dropout(B.F32, N, C, x, p, state(seed, step), layer, y)
        keep = kept(N, C, p, seed, step, layer)
        got = y.cpu().numpy()
        assert (got[~keep] == 0).all() and np.array_equal(np.isnan(got[:, 1::2]), keep[:, 1::2]) and np.array_equal(np.isinf(got[:, ::2]), keep[:, ::2])
        masks.append(keep)
    for i in range(len(masks)):
        for j in range(i):
            assert 0.4 < (masks[i] == masks[j]).mean() < 0.6       # independent halves agree on half of 4000: 0.5 +- 0.05 is 6 sigma


class Norm:
    def __init__(self, dtype, N, C, seed, ldx=None, ldy=None, p=0.0, relu=False, offset=1.0, gamma=True, beta=True, g_dtype=None, layer=3):
        rng = np.random.default_rng(seed)
        self.dtype, self.g_dtype, self.N, self.C, self.p, self.relu, self.layer = dtype, dtype if g_dtype is None else g_dtype, N, C, p, relu, layer
        self.ldx, self.ldy = C if ldx is None else ldx, C if ldy is None else ldy
        f32 = lambda a: torch.from_numpy(a.astype(np.float32))  # noqa: E731
        x = f32(rng.standard_normal((N, C)) * (0.5 + rng.random((N, 1))) + offset * rng.standard_normal((N, 1)))
        self.x = (x.clamp_min(0) if relu else x).to(TDT[dtype])
        self.dy = f32(rng.standard_normal((N, C))).to(TDT[self.g_dtype])
        self.gamma = f32(1 + 0.3 * rng.standard_normal(C)) if gamma else None
        self.beta = f32(0.2 * rng.standard_normal(C)) if beta else None
        self.seed, self.step = 77 + seed, 9
        self.rng = state(self.seed, self.step) if p else None
        self.xs = padded(self.x, self.ldx, dtype)
        self.cuda = lambda t: None if t is None else t.cuda()
        self.gd, self.bd = self.cuda(self.gamma), self.cuda(self.beta)

    def forward(self, y=None):
        self.y = torch.full((self.N, self.ldy), 3.0, dtype=TDT[self.dtype], device="cuda") if y is None else y
        self.stats = torch.full((self.N, 2), 3.0, device="cuda")
        B.vgg_layer_norm(self.dtype, self.N, self.C, self.xs, self.gd, self.bd, EPS, self.p, self.rng, self.layer, self.y, self.stats, ldx=self.ldx, ldy=self.ldy)
        return self

    def backward(self, in_place=False, want=(True, True)):
        lddy, lddx = self.ldy, self.ldy if in_place else self.ldx
        dy = padded(self.dy, lddy, self.g_dtype)
        self.dx = dy if in_place else torch.full((self.N, lddx), 3.0, dtype=TDT[self.g_dtype], device="cuda")
        self.dgamma, self.dbeta = (torch.full((self.C,), 3.0, device="cuda") if w else None for w in want)
        ws = ws_bytes(B.vgg_layer_norm_bwd_workspace_bytes(self.dtype, self.g_dtype, self.N, self.C))
        ws.fill_(0xFF)
        B.vgg_layer_norm_bwd(self.dtype, self.g_dtype, self.N, self.C, self.xs, self.gd, self.stats, self.p, self.rng, self.layer, dy, self.dx, self.dgamma,
                             self.dbeta, self.relu, ws, ldx=self.ldx, lddy=lddy, lddx=lddx)
        return self

    def reference(self):
        x, dy = self.x.double(), self.dy.double()
        mean = x.mean(1, keepdim=True)
        rstd = 1 / ((x - mean).square().mean(1, keepdim=True) + EPS).sqrt()
        xh = (x - mean) * rstd
        gamma = torch.ones(self.C, dtype=torch.float64) if self.gamma is None else self.gamma.double()
        beta = torch.zeros(self.C, dtype=torch.float64) if self.beta is None else self.beta.double()
        f = torch.from_numpy(kept(self.N, self.C, self.p, self.seed, self.step, self.layer)) * scale(self.p) if self.p else torch.ones(())
        g = dy * f
        gg = g * gamma
        dx = rstd * (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True))
        if self.relu:
            dx = torch.where(x > 0, dx, 0.0)
        # How far fp32 arithmetic may be off.  A thread adds up to 32 values, then sums go through at most 12 additions and a division: means are off by
        # up to 48 u of the mean magnitude; a difference from the mean by 50 u of the largest one, X in units of the width; xh by that and the
        # relative error of the width, half of 48 u and what the mean's shift leaves of it.
        X = x.abs().amax(1, keepdim=True) * rstd
        e_xh = 60 * U * (X + xh.abs())
        tol = {"y": f * (gamma.abs() * e_xh + 4 * U * (xh * gamma).abs() + 2 * U * beta.abs())}
        m1, m2 = gg.abs().mean(1, keepdim=True), (gg.abs() * (xh.abs() + e_xh)).mean(1, keepdim=True)
        tol["dx"] = rstd * (64 * U * (gg.abs() + m1 + xh.abs() * m2) + e_xh * m2 + xh.abs() * (gg.abs() * e_xh).mean(1, keepdim=True)) + 60 * U * dx.abs()
        # a column's sums: a term to a row in turn, N at most, and the parts'
        tol["dbeta"] = (self.N + 40) * U * g.abs().sum(0)
        tol["dgamma"] = (self.N + 40) * U * (g * xh).abs().sum(0) + (g.abs() * e_xh).sum(0)
        tol["y"] = tol["y"] + HALF[self.dtype] * (xh * gamma + beta).abs() * f
        tol["dx"] = tol["dx"] + HALF[self.g_dtype] * dx.abs()
        return {"y": (xh * gamma + beta) * f, "mean": mean[:, 0], "rstd": rstd[:, 0], "dx": dx, "dgamma": (g * xh).sum(0), "dbeta": g.sum(0)}, tol

    def check(self, back=True):
        torch.cuda.synchronize()
        want, tol = self.reference()
        C = self.C
        near = lambda got, name: (((got.double().cpu() - want[name]).abs() <= tol[name] + 1e-30).all(), name,  # noqa: E731
                                  ((got.double().cpu() - want[name]).abs() - tol[name]).max())
        ok = [near(self.y[:, :C], "y")]
        assert (self.y[:, C:] == 3.0).all()
        x = self.x.double()
        assert ((self.stats[:, 0].double().cpu() - want["mean"]).abs() <= 48 * U * x.abs().amax(1)).all()
        big = x.abs().amax(1) * want["rstd"]
        assert ((self.stats[:, 1].double().cpu() / want["rstd"] - 1).abs() <= 60 * U * (1 + 48 * U * big * big)).all()
        if back:
            ok.append(near(self.dx[:, :C], "dx"))
            ok += [near(t, n) for t, n in ((self.dgamma, "dgamma"), (self.dbeta, "dbeta")) if t is not None]
        for good, name, over in ok:
            assert good, (name, float(over))


TYPES = [(B.F32, B.F32), (B.BF16, B.BF16), (B.BF16, B.F32)]
# a team of every size, its last column alone and the first past it; rows that fill no team's workgroup
SIZES = [(1, 1), (2, 8), (33, 9), (65, 64), (40, 65), (17, 128), (9, 129), (19, 256), (5, 257), (301, 333), (4, 512), (6, 513), (3, 1000), (2, 1024), (3, 1025), (2, 2048), (5, 2049),
         (100, 4096), (3, 4097), (2, 8191), (3, 8193), (2, 16384), (3, 16385), (4, 25088), (2, 28672), (3, 28673), (2, 70001)]


@pytest.mark.parametrize("dtype,g_dtype", TYPES)
@pytest.mark.parametrize("N,C", SIZES)
def test_layer_norm_and_gradient(dtype, g_dtype, N, C):
    Norm(dtype, N, C, N + C, g_dtype=g_dtype, p=0.5 if C % 2 else 0.0, relu=C % 3 == 0).forward().backward().check()


@pytest.mark.parametrize("dtype,g_dtype", TYPES)
@pytest.mark.parametrize("N,C", [(3000, 40), (5000, 700), (700, 5000), (300, 25088), (2500, 2)])
def test_more_rows_than_run_at_once(dtype, g_dtype, N, C):
    Norm(dtype, N, C, 5, g_dtype=g_dtype, p=0.1).forward().backward().check()


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("N,C,ldx,ldy", [(7, 333, 336, 333), (9, 333, 334, 341), (5, 4096, 4097, 4099), (3, 40000, 40001, 40003)])
def test_strides_and_missing_vectors(dtype, N, C, ldx, ldy):
    Norm(dtype, N, C, 1, ldx=ldx, ldy=ldy, p=0.25, relu=True).forward().backward().check()
    Norm(dtype, N, C, 2, ldx=ldx, ldy=ldy, gamma=False, beta=False).forward().backward(want=(True, False)).check()
    Norm(dtype, N, C, 3, ldx=ldx, ldy=ldy, gamma=False).forward().backward(want=(False, True), in_place=True).check()
    Norm(dtype, N, C, 4, ldx=ldx, ldy=ldy, beta=False).forward().backward(want=(False, False)).check()


@pytest.mark.parametrize("C", [64, 700, 4096, 20000, 40000])
def test_rows_far_from_zero_and_constant_rows(C):
    Norm(B.F32, 5, C, 6, offset=1000.0).forward().backward().check()
    n = Norm(B.F32, 4, C, 7)
    n.x[:] = torch.tensor([0.0, 3.0, -1e-3, 1e4])[:, None]
    n.xs = padded(n.x, C, B.F32)
    n.forward().backward()
    torch.cuda.synchronize()
    # a mean of equal values is off by up to 48 u of them, xh by that over the square root of eps
    off = 50 * U * n.x.abs().double() / EPS ** 0.5
    assert ((n.y.double().cpu() - n.beta.double()).abs() <= off * n.gamma.abs().double() + U).all()
    assert torch.isfinite(n.dx).all()


def test_nan_stays_in_its_row():
    n = Norm(B.BF16, 6, 1000, 8, p=0.5)
    n.x[2, 17], n.x[4, 3] = float("nan"), float("inf")
    n.xs = padded(n.x, n.ldx, n.dtype)
    n.forward().backward()
    keep = torch.from_numpy(kept(6, 1000, 0.5, n.seed, n.step, n.layer))
    y, dx = n.y.cpu(), n.dx.cpu()
    for row in (2, 4):
        assert torch.isnan(y[row][keep[row]]).all() and (y[row][~keep[row]] == 0).all() and torch.isnan(dx[row]).all()
    rest = [0, 1, 3, 5]
    assert torch.isfinite(y[rest].float()).all() and torch.isfinite(dx[rest].float()).all()


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("C", [50, 4096, 25088, 33000])
def test_in_place_dropout_apart_and_twice_the_same(dtype, C):
    n = Norm(dtype, 6, C, 9, p=0.5, relu=True)
    n.forward().backward()
    y, dx, dgamma = n.y.clone(), n.dx.clone(), n.dgamma.clone()
    n.forward().backward()
    assert torch.equal(y, n.y) and torch.equal(dx, n.dx) and torch.equal(dgamma, n.dgamma)
    n.backward(in_place=True)     # (few rows: dgamma's six terms are added in another order, each way within check()'s bound)
    assert torch.equal(dx, n.dx)
    n.check()
    if dtype == B.F32:            # the fused dropout is that of vgg_dropout
        apart, drop = Norm(dtype, 6, C, 9, relu=True), torch.empty_like(y)
        apart.forward()
        B.vgg_dropout(dtype, 6, C, apart.y, 0.5, n.rng, n.layer, drop)
        assert torch.equal(drop, y)
    x0 = n.xs.clone()
    n.forward(y=n.xs)
    assert torch.equal(n.xs, y)
    n.xs = x0
    # the gradient where the activations were
    dy = padded(n.dy, C, dtype)
    ws = ws_bytes(B.vgg_layer_norm_bwd_workspace_bytes(dtype, dtype, 6, C))
    B.vgg_layer_norm_bwd(dtype, dtype, 6, C, n.xs, n.gd, n.stats, 0.5, n.rng, n.layer, dy, n.xs, None, None, True, ws)
    assert torch.equal(n.xs, dx)


def test_gradient_against_differences():
    # fp32 forward in 64-bit steps is not to be had: the loss's slope along a direction, by differences of the 64-bit definition at the kernel's inputs
    n = Norm(B.F32, 5, 37, 10, p=0.25).forward().backward()
    rng = np.random.default_rng(1)
    f = torch.from_numpy(kept(5, 37, 0.25, n.seed, n.step, n.layer)) * scale(0.25)

    def loss(x, gamma, beta):
        mean = x.mean(1, keepdim=True)
        return (((x - mean) / ((x - mean).square().mean(1, keepdim=True) + EPS).sqrt() * gamma + beta) * f * n.dy.double()).sum()

    at = (n.x.double(), n.gamma.double(), n.beta.double())
    for i, grad in enumerate((n.dx, n.dgamma, n.dbeta)):
        way = torch.from_numpy(rng.standard_normal(at[i].shape))
        h = 1e-5
        step = [loss(*[t + s * h * way if k == i else t for k, t in enumerate(at)]) for s in (1, -1)]
        slope, got = (step[0] - step[1]) / (2 * h), (grad.double().cpu() * way).sum()
        # second differences leave h^2 of a third derivative, some 1e-9; fp32 gradients 1e-6 of the sum of magnitudes
        assert abs(slope - got) <= 1e-5 * (grad.double().cpu() * way).abs().sum() + 1e-6


def test_another_stream_and_a_graph_that_drops_anew():
    N, C, p = 64, 700, 0.5
    n = Norm(B.BF16, N, C, 11, p=p)
    n.forward().backward()
    y, dx, dgamma = n.y.clone(), n.dx.clone(), n.dgamma.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        n.forward().backward()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, n.y) and torch.equal(dx, n.dx) and torch.equal(dgamma, n.dgamma)
    out, dxo, dg, db = torch.empty_like(y), torch.empty_like(dx), torch.empty_like(dgamma), torch.empty_like(dgamma)
    dy = padded(n.dy, C, B.BF16)
    ws = ws_bytes(B.vgg_layer_norm_bwd_workspace_bytes(B.BF16, B.BF16, N, C))

    def step():
        B.vgg_layer_norm(B.BF16, N, C, n.xs, n.gd, n.bd, EPS, p, n.rng, 3, out, n.stats)
        B.vgg_layer_norm_bwd(B.BF16, B.BF16, N, C, n.xs, n.gd, n.stats, p, n.rng, 3, dy, dxo, dg, db, False, ws)
        n.rng[1] += 1

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(4):
        n.step = int(n.rng[1])
        out.fill_(5), dg.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert int(n.rng[1]) == n.step + 1
        n.y, n.dx, n.dgamma, n.dbeta = out, dxo, dg, db
        n.check()
