"""Orthogonalised updates against Newton-Schulz in 64 bits: both operand precisions, shapes that fill no tile, tall and wide,
batches, special values, and the optimiser step around them."""
import numpy as np
import pytest
import torch

from paper_1810_09868_amd import binding as B

from gpu_util import TDT, ws_bytes
from plan_shapes import MUON_256

pytestmark = pytest.mark.gpu

COEFF = (3.4445, -4.7750, 2.0315)


def ns64(u, steps):
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (np.sqrt((x * x).sum()) + 1e-7)
    for _ in range(steps):
        g = x @ x.T
        x = COEFF[0] * x + (COEFF[1] * g + COEFF[2] * (g @ g)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def matrices(dtype, batch, rows, cols, seed, kind="gradient"):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((batch, rows, cols))
    if kind == "gradient":                        # a few strong directions over noise
        for b in range(batch):
            x[b] = 0.05 * x[b] + rng.standard_normal((rows, 4)) @ np.abs(rng.standard_normal((4, cols)))
    return torch.from_numpy(x.astype(np.float32)).to(TDT[dtype])


def orthogonalize(dtype, x, steps, in_place=False):
    batch, rows, cols = x.shape
    x = x.cuda()
    y = x if in_place else torch.full_like(x, float("nan"))
    ws = ws_bytes(B.vgg_orthogonalize_workspace_bytes(dtype, batch, rows, cols))
    ws.fill_(0xFF)                                # NaN wherever it is read before it is written
    B.vgg_orthogonalize(dtype, batch, rows, cols, steps, x, y, ws)
    torch.cuda.synchronize()
    return y.cpu().double().numpy()


# 2-norm of the difference over that of the result.  fp32: a rounding of X (2^-24) grows 3.4445-fold a step where the singular
# values are small, 485-fold over five steps; products are as exact as fp32's.  485 x 2^-24 = 2.9e-5 is the bound.  bf16: its own
# rounding is 2^-9 / sqrt(3) x 1.5 (mean square over a binade) = 1.7e-3; operands of 11 bits add up to 1e-3 by the simulation
# that the kernel's comment cites: 3e-3 in all, one step less of both.
def bound(dtype):
    return 3e-5 if dtype == B.F32 else 3e-3


def off(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


SHAPES = [(1, 1, 1), (1, 1, 37), (2, 37, 1), (1, 2, 3), (3, 16, 16), (1, 27, 64), (2, 64, 27), (1, 64, 576), (1, 127, 129), (1, 129, 127), (1, 130, 514),
          (2, 200, 1000), (1, 1000, 200), (1, 255, 257), (1, 300, 300), (3, 96, 33), (2, 33, 480), (1, 481, 64), (1, 64, 768), (1, 769, 40), (1, 65, 100), (5, 32, 32)]


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize_against_64_bits(dtype, shape):
    for kind, steps in (("gradient", 5), ("noise", 5), ("noise", 1)):
        x = matrices(dtype, *shape, seed=sum(shape) + steps, kind=kind)
        got = orthogonalize(dtype, x, steps)
        for b in range(shape[0]):
            e = off(got[b], ns64(x[b].double().numpy(), steps))
            assert e <= bound(dtype), (shape, kind, steps, b, e)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", [(1, 512, 4608), (1, 1000, 4096), (7, 256, 2304), (1, 2100, 700), (3, 989, 16), (2, 28, 7933), (1, 64, 4097), (1, 30000, 10), (5, 3209, 64), (1, 1300, 5000), (2, 2048, 2048)])
def test_orthogonalize_of_the_networks_shapes(dtype, shape):
    x = matrices(dtype, *shape, seed=1)
    got = orthogonalize(dtype, x, 5)
    for b in range(shape[0]):
        u = x[b].double().cuda()
        u = u.t() if shape[1] > shape[2] else u
        u = u / (torch.linalg.vector_norm(u) + 1e-7)
        for _ in range(5):
            g = u @ u.t()
            u = COEFF[0] * u + COEFF[1] * (g @ u) + COEFF[2] * (g @ (g @ u))
        want = (u.t() if shape[1] > shape[2] else u).cpu().numpy()
        e = off(got[b], want)
        assert e <= bound(dtype), (b, e)


def test_singular_values_come_near_one():
    x = matrices(B.F32, 1, 200, 333, 3, "noise")
    s = np.linalg.svd(orthogonalize(B.F32, x, 5)[0], compute_uv=False)
    assert s.max() < 1.25 and np.median(s) > 0.65


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_in_place_and_the_same_every_time(dtype):
    x = matrices(dtype, 2, 130, 300, 5)
    a = orthogonalize(dtype, x, 5)
    assert np.array_equal(a, orthogonalize(dtype, x, 5, in_place=True)) and np.array_equal(a, orthogonalize(dtype, x, 5))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_matrices_of_a_batch_do_not_meet(dtype):
    x = matrices(dtype, 5, 70, 150, 6)
    x[1] = 0
    x[2, 3, 4] = float("nan")
    x[3, 60, 140] = float("inf")
    got = orthogonalize(dtype, x, 5)
    assert not got[1].any() and np.isnan(got[2]).all() and np.isnan(got[3]).all()
    for b in (0, 4):
        assert off(got[b], ns64(x[b].double().numpy(), 5)) <= bound(dtype)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -20, 2.0 ** 20, 2.0 ** 100, 2.0 ** 118])
def test_scale_of_the_input(dtype, scale):
    # 1e-7 beside the norm counts for small matrices only
    x = matrices(dtype, 1, 40, 60, 8)
    got = orthogonalize(dtype, x * scale, 5)
    want = ns64(x[0].double().numpy() * scale, 5)
    assert off(got[0], want) <= bound(dtype)


def test_a_matrix_of_one_direction():
    # every other singular value is rounding, which each step enlarges: fp32 torch products are 1e-4 off here
    rng = np.random.default_rng(2)
    x = torch.from_numpy(np.outer(rng.standard_normal(150), rng.standard_normal(260)).astype(np.float32))[None]
    for dtype in (B.F32, B.BF16):
        s = np.linalg.svd(orthogonalize(dtype, x.to(TDT[dtype]), 5)[0], compute_uv=False)
        assert 0.65 < s[0] < 1.25
    want = ns64(x[0].double().numpy(), 5)
    u = x[0].cuda()
    u = u / (u.square().sum().sqrt() + 1e-7)
    for _ in range(5):
        g = u @ u.t().contiguous()
        u = COEFF[0] * u + (COEFF[1] * g + COEFF[2] * (g @ g)) @ u
    assert off(orthogonalize(B.F32, x, 5)[0], want) <= off(u.double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(1, 10, 512), (2, 300, 100), (1, 1000, 513)])
def test_update_against_64_bits(dtype, nesterov, shape):
    rng = np.random.default_rng(sum(shape))
    theta, m0 = (rng.standard_normal(shape).astype(np.float32) for _ in range(2))
    lr, mu, decay, steps = 0.05, 0.9, 0.1, 5
    t, m = torch.from_numpy(theta).cuda(), torch.from_numpy(m0).cuda()
    ws = ws_bytes(B.vgg_muon_workspace_bytes(dtype, *shape))
    want_t, want_m = theta.astype(np.float64), m0.astype(np.float64)
    for k in range(3):
        g = matrices(B.F32, *shape, seed=k)
        B.vgg_muon_update(dtype, *shape, steps, t, g.cuda(), m, lr, mu, nesterov, decay, ws)
        g = g.double().numpy()
        want_m = mu * want_m + g
        for b in range(shape[0]):
            o = ns64(g[b] + mu * want_m[b] if nesterov else want_m[b], steps)
            want_t[b] = (1 - lr * decay) * want_t[b] - lr * np.sqrt(max(1, shape[1] / shape[2])) * o
    torch.cuda.synchronize()
    assert off(m.cpu().numpy(), want_m) < 3e-7                    # a few fp32 roundings
    step = 3 * lr * np.sqrt(max(1, shape[1] / shape[2]))          # what three updates can be off
    allow = step * bound(dtype) * np.linalg.norm(o) + 1e-6 * np.linalg.norm(want_t)
    assert np.linalg.norm(t.cpu().numpy() - want_t) <= allow * np.sqrt(shape[0])


def test_refusals():
    a = torch.zeros((1 << 16,), device="cuda")
    ok = dict(dtype=B.F32, batch=1, rows=8, cols=8, steps=5, x=a, y=a, ws=a.new_zeros((1 << 22,)))
    for change, status in [(dict(x=None), -1), (dict(y=None), -1), (dict(dtype=3), -3), (dict(batch=0), -2), (dict(rows=0), -2), (dict(cols=-1), -2),
                           (dict(steps=0), -2), (dict(steps=21), -2), (dict(rows=40000, cols=40000), -2), (dict(batch=70000), -2), (dict(ws=None), -5),
                           (dict(ws=a[:64]), -5), (dict(x=a[1:]), -4)]:
        with pytest.raises(B.VggError) as e:
            B.vgg_orthogonalize(**{**ok, **change})
        assert e.value.status == status, change
    with pytest.raises(B.VggError) as e:
        B.vgg_muon_update(B.F32, 1, 8, 8, 5, a, a, None, 0.1, 0.9, True, 0.0, ok["ws"])
    assert e.value.status == -1
    assert B.vgg_muon_workspace_bytes(B.F32, 1, 0, 8) == 0 and B.vgg_orthogonalize_workspace_bytes(9, 1, 8, 8) == 0


def test_on_another_stream_and_in_a_graph():
    x = matrices(B.F32, 1, 140, 400, 4).cuda()
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    ws = ws_bytes(B.vgg_orthogonalize_workspace_bytes(B.F32, 1, 140, 400))
    call = lambda out: B.vgg_orthogonalize(B.F32, 1, 140, 400, 5, x, out, ws)  # noqa: E731
    call(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(z)
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(z)
    for k in range(3):
        x.copy_(matrices(B.F32, 1, 140, 400, 40 + k))
        call(y)
        z.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, z), k


def ns64_gpu(u, steps):
    x = u.t().contiguous() if u.shape[0] > u.shape[1] else u
    x = x / (torch.linalg.vector_norm(x) + 1e-7)
    for _ in range(steps):
        g = x @ x.t().contiguous()
        x = COEFF[0] * x + COEFF[1] * (g @ x) + COEFF[2] * (g @ (g @ x))
    return x.t() if u.shape[0] > u.shape[1] else x


# A bf16 result that is off by a relative e before it is rounded is another bf16 number than the rounded exact value with
# probability |error| / spacing, and then a spacing (at most 2^-7 of the value) off: a mean square of at most e 2^-7 of the values'.
# e is fp32's bound; operands of 11 bits (e some 5e-4 to 1.6e-3) are 1.3e-3 off and more by this measure.
@pytest.mark.parametrize("kind", ["gradient", "noise"])
@pytest.mark.parametrize("shape", [(1, 64, 576), (1, 40, 300), (2, 50, 2000), (1, 130, 514), (1, 2100, 130), (2, 512, 4608)])
def test_bf16_results_are_exact_ones_rounded(shape, kind):
    x = matrices(B.BF16, *shape, seed=11, kind=kind)
    got = orthogonalize(B.BF16, x, 5)
    for b in range(shape[0]):
        want = ns64_gpu(x[b].double().cuda(), 5).to(torch.bfloat16).double().cpu().numpy()
        assert off(got[b], want) <= np.sqrt(2.0 ** -7 * bound(B.F32)) + bound(B.F32)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("scale", [2.0 ** -110, 2.0 ** -64, 2.0 ** -50, 2.0 ** -40, 2.0 ** -30])
@pytest.mark.parametrize("shape", [(40, 60), (50, 1500), (130, 514), (300, 130)])
def test_matrices_whose_norm_is_small_beside_the_added_constant(dtype, scale, shape):
    # X_0 is then small itself and grows 3.4445-fold a step: no fixed scale holds its digits
    x = matrices(dtype, 1, *shape, seed=9) * scale
    assert off(orthogonalize(dtype, x, 5)[0], ns64(x[0].double().numpy(), 5)) <= bound(dtype)
    g = x.float().cuda()
    theta, mom = torch.zeros_like(g), torch.zeros_like(g)
    B.vgg_muon_update(dtype, 1, *shape, 5, theta, g, mom, 1.0, 0.9, False, 0.0, ws_bytes(B.vgg_muon_workspace_bytes(dtype, 1, *shape)))
    want = -np.sqrt(max(1, shape[0] / shape[1])) * ns64(x[0].double().numpy(), 5)
    assert off(theta[0].double().cpu().numpy(), want) <= bound(dtype)


def on_gpu(dtype, shape, seed):
    """matrices(), drawn on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = torch.stack([0.05 * normal(*shape[1:]) + normal(shape[1], 4) @ normal(4, shape[2]).abs() for _ in range(shape[0])])
    return x.to(TDT[dtype])


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", MUON_256)
def test_orthogonalize_by_the_largest_tiles(dtype, shape):
    x = on_gpu(dtype, shape, 5)
    y = torch.full_like(x, float("nan"))
    ws = ws_bytes(B.vgg_orthogonalize_workspace_bytes(dtype, *shape))
    ws.fill_(0xFF)
    B.vgg_orthogonalize(dtype, *shape, 5, x, y, ws)
    for b in range(shape[0]):
        want = ns64_gpu(x[b].double(), 5)
        assert float((y[b].double() - want).norm() / want.norm()) <= bound(dtype)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", MUON_256[1:])
def test_update_by_the_largest_tiles(dtype, shape):
    lr, mu, decay = 0.05, 0.9, 0.1
    theta, m = (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda") for k in (1, 2))
    ws = ws_bytes(B.vgg_muon_workspace_bytes(dtype, *shape))
    want_t, want_m = theta.double(), m.double()
    for k in range(2):
        g = on_gpu(B.F32, shape, 10 + k)
        ws.fill_(0xFF)
        B.vgg_muon_update(dtype, *shape, 5, theta, g, m, lr, mu, True, decay, ws)
        want_m = mu * want_m + g.double()
        o = torch.stack([ns64_gpu(u, 5) for u in g.double() + mu * want_m])
        want_t = (1 - lr * decay) * want_t - lr * max(1.0, shape[1] / shape[2]) ** 0.5 * o
    assert float((m.double() - want_m).norm() / want_m.norm()) < 3e-7
    allow = 2 * lr * max(1.0, shape[1] / shape[2]) ** 0.5 * bound(dtype) * float(o.norm()) + 1e-6 * float(want_t.norm())
    assert float((theta.double() - want_t).norm()) <= allow


def test_matrices_of_the_largest_tiles_do_not_meet():
    shape = (4, 1270, 2500)
    x = on_gpu(B.BF16, shape, 3)
    x[1] = 0
    x[2, 700, 2400] = float("nan")
    alone = torch.empty_like(x)
    ws = ws_bytes(B.vgg_orthogonalize_workspace_bytes(B.BF16, *shape))
    B.vgg_orthogonalize(B.BF16, *shape, 5, x, alone, ws)
    again = x.clone()
    B.vgg_orthogonalize(B.BF16, *shape, 5, again, again, ws)
    assert not alone[1].any() and alone[2].isnan().all()
    for b in (0, 3):
        assert torch.equal(alone[b], again[b])
        want = ns64_gpu(x[b].double(), 5)
        assert float((alone[b].double() - want).norm() / want.norm()) <= bound(B.BF16)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", [(1, 40, 200001), (2, 140001, 17), (1, 1, 250000), (1, 64, 114700)])
def test_few_rows_and_very_many_columns(dtype, shape):
    # about where one launch a step ends and tiles begin, and beyond
    x = on_gpu(dtype, shape, 21)
    y = torch.full_like(x, float("nan"))
    ws = ws_bytes(B.vgg_orthogonalize_workspace_bytes(dtype, *shape))
    ws.fill_(0xFF)
    B.vgg_orthogonalize(dtype, *shape, 5, x, y, ws)
    theta, mom, g = torch.zeros_like(y, dtype=torch.float32), torch.zeros_like(y, dtype=torch.float32), x.float()
    B.vgg_muon_update(dtype, *shape, 5, theta, g, mom, 1.0, 0.9, False, 0.0, ws)
    scale = max(1.0, shape[1] / shape[2]) ** 0.5
    for b in range(shape[0]):
        want = ns64_gpu(x[b].double(), 5)
        assert float((y[b].double() - want).norm() / want.norm()) <= bound(dtype)
        assert float((theta[b].double() / -scale - want).norm() / want.norm()) <= bound(dtype)
