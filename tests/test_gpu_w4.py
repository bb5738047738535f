"""Dense layers from 4-bit weights: codes and scales against exact rounding, products against the dequantised weights in 64
bits, at sizes that fill no group, block or tile, over every path (a few rows, tiles of rows, split inputs)."""
import numpy as np
import pytest
import torch

from paper_1810_09868_amd import binding as B

from gpu_util import TDT, ws_bytes
from plan_shapes import W4_TILES

pytestmark = pytest.mark.gpu

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def buffers(In, Out, group):
    codes = torch.full((Out, -(-In // 32) * 16), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((Out, -(-In // group)), 3.0, dtype=torch.bfloat16, device="cuda")
    return codes, scales


def quantize64(w, group):
    """(values, scales) by the definition, in numpy's 64 bits: nearest value by trial, the even code at ties."""
    Out, In = w.shape
    v, sc = np.zeros((Out, In)), np.zeros((Out, -(-In // group)))
    for j in range(0, In, group):
        g = w[:, j:j + group]
        most = np.abs(g).max(1).astype(np.float32) * np.float32(1 / 6)
        s = torch.from_numpy(most).to(torch.bfloat16).double().numpy()
        sc[:, j // group] = s
        d = np.abs(np.abs(g.astype(np.float64))[:, :, None] - s[:, None, None] * GRID)
        best = d.min(2, keepdims=True)
        near = d == best
        code = np.where(near[:, :, 0::2].any(2), 2 * near[:, :, 0::2].argmax(2), near.argmax(2))
        v[:, j:j + group] = np.sign(g) * GRID[code] * s[:, None]
    return v, sc


def weights(In, Out, seed):
    return (np.random.default_rng(seed).standard_normal((Out, In)) * np.sqrt(2.0 / In)).astype(np.float32)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("In,Out", [(1, 1), (31, 3), (32, 5), (33, 7), (127, 2), (128, 9), (129, 33), (1000, 10), (4096, 65)])
def test_quantize_is_exact_rounding(In, Out, group):
    w = weights(In, Out, In + group)
    w[0, : min(In, 40)] = (np.arange(min(In, 40)) - 20) * 0.25      # ties of every kind, where the scale is a power of two
    w[0, 0] = 6.0
    if Out > 1:
        w[1, :] = 0.0
    codes, scales = buffers(In, Out, group)
    out = torch.full((Out, In), float("nan"), device="cuda")
    B.vgg_fc_w4_quantize(In, Out, group, torch.from_numpy(w).cuda(), codes, scales)
    B.vgg_fc_w4_dequantize(In, Out, group, codes, scales, out)
    torch.cuda.synchronize()
    v, sc = quantize64(w, group)
    assert np.array_equal(scales.double().cpu().numpy(), sc)
    assert np.array_equal(out.double().cpu().numpy(), v)
    pad = torch.stack((codes & 15, codes >> 4), 2).flatten(1)[:, In:]
    assert int(pad.sum()) == 0


def test_quantize_marks_a_group_that_is_not_finite_and_no_other():
    w = weights(256, 4, 3)
    w[1, 5], w[2, 70], w[3, 255] = np.nan, np.inf, -np.inf
    codes, scales = buffers(256, 4, 64)
    out = torch.zeros((4, 256), device="cuda")
    B.vgg_fc_w4_quantize(256, 4, 64, torch.from_numpy(w).cuda(), codes, scales)
    B.vgg_fc_w4_dequantize(256, 4, 64, codes, scales, out)
    torch.cuda.synchronize()
    bad = np.zeros((4, 4), bool)
    bad[1, 0] = bad[2, 1] = bad[3, 3] = True
    assert np.array_equal(torch.isnan(scales).cpu().numpy(), bad)
    assert np.array_equal(torch.isnan(out).cpu().numpy(), bad.repeat(64, 1))


def test_dequantize_of_every_code():
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(1, 256).contiguous()
    scales = torch.full((1, 4), 0.75, dtype=torch.bfloat16, device="cuda")
    out = torch.empty((1, 512), device="cuda")
    B.vgg_fc_w4_dequantize(512, 1, 128, codes, scales, out)
    both = np.stack((np.arange(256) & 15, np.arange(256) >> 4), 1).reshape(-1)
    want = GRID[both & 7] * np.where(both & 8, -0.75, 0.75)
    assert np.array_equal(out.double().cpu().numpy()[0], want)


def product(dtype, N, In, Out, group, relu, zdt, seed, bias=True, special=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (Out, -(-In // 32) * 16), generator=g, device="cuda", dtype=torch.uint8)   # padding codes too
    scales = (torch.rand((Out, -(-In // group)), generator=g, device="cuda") * 0.02 + 1e-3).to(torch.bfloat16)
    a = torch.randn((N, In), generator=g, device="cuda").to(TDT[dtype])
    if special:
        special(a, scales)
    b = torch.randn((Out,), generator=g, device="cuda") if bias else None
    z = torch.full((N, Out), float("nan"), dtype=TDT[zdt], device="cuda")
    ws = ws_bytes(B.vgg_fc_w4_workspace_bytes(dtype, N, In, Out, group))
    ws.fill_(0xFF)
    B.vgg_fc_w4(dtype, N, In, Out, group, a, codes, scales, b, z, zdt, relu, ws)
    torch.cuda.synchronize()
    nib = torch.stack((codes & 15, codes >> 4), 2).flatten(1)[:, :In].cpu()
    w = torch.from_numpy(GRID)[(nib & 7).long()] * torch.where(nib >= 8, -1.0, 1.0).double()
    w = w * scales.double().cpu().repeat_interleave(group, 1)[:, :In]
    a64 = a.double().cpu()
    want = a64 @ w.t() + (0 if b is None else b.double().cpu())
    size = a64.abs() @ w.abs().t() + (0 if b is None else b.double().cpu().abs())
    if relu:
        want = torch.where(want < 0, 0.0, want)
    return z.double().cpu(), want, size


# A result's error: an fp32 sum of In products, each exact, added in runs of at most In/32 (a few dozen sequential additions of
# 2^-24 each relative to the sum of magnitudes; the matrix unit cuts off what it aligns, 2^-23): 64 x 2^-23 = 7.7e-6 of that sum
# is never reached.  bf16 results add half of 2^-8.
def check(got, want, size, zdt):
    assert torch.isfinite(got).all()
    err = (got - want).abs()
    allow = 7.7e-6 * size + (2.0 ** -8 * want.abs() if zdt == B.BF16 else 0)
    assert (err <= allow).all(), float((err / size).max())


SHAPES = [(1, 1), (7, 3), (31, 16), (32, 17), (64, 10), (127, 33), (129, 5), (136, 40), (512, 100), (1000, 63), (2047, 20), (2049, 9), (4096, 130)]


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 16, 17, 32, 33, 64, 65, 130])
def test_product_against_64_bits(dtype, N):
    for k, (In, Out) in enumerate(SHAPES):
        group = (32, 64, 128)[(k + N) % 3]
        zdt = dtype if k % 2 else B.F32
        check(*product(dtype, N, In, Out, group, relu=(k + N) % 2 == 0, zdt=zdt, seed=100 * k + N, bias=k % 3 != 0), zdt)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N", [1, 10, 20, 100])
def test_product_of_the_networks_layers(dtype, group, N):
    check(*product(dtype, N, 4096, 1000, group, False, B.F32, seed=N + group), B.F32)


@pytest.mark.parametrize("N", [1, 4, 12, 70])
def test_product_of_a_long_row(N):
    check(*product(B.BF16, N, 40001, 24, 128, True, B.F32, seed=N), B.F32)
    check(*product(B.F32, N, 33000, 24, 32, False, B.F32, seed=N), B.F32)


def test_product_is_the_same_every_time():
    a = [product(B.BF16, 100, 4096, 256, 64, True, B.F32, seed=5)[0] for _ in range(3)]
    assert torch.equal(a[0], a[1]) and torch.equal(a[0], a[2])


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("N", [1, 3, 9, 40, 80])
def test_infinities_and_nans_stay_where_they_belong(dtype, N):
    In, Out, group = 160, 24, 32
    row = N - 1

    def special(a, scales):
        a[row, 70] = float("inf")                # every output of this row is infinite or, where the code is 0, NaN
        scales[5, 4] = float("nan")              # output 5 of every row

    got, want, _ = product(dtype, N, In, Out, group, False, B.F32, seed=N, special=special)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert inf.any() and torch.equal(got[inf], want[inf])
    rest = torch.isfinite(want)
    assert not rest.any() or (got[rest] - want[rest]).abs().max() <= 1e-4 * want[rest].abs().max()   # (one row: none is finite)


def test_large_activations_do_not_overflow_in_parts():
    def special(a, scales):
        a[0, 3] = 3.3e38
        scales.fill_(2.0 ** -10)

    for N in (1, 6):
        got, want, size = product(B.F32, N, 64, 20, 32, False, B.F32, seed=N, special=special)
        assert ((got - want).abs() <= 1e-5 * size).all()


def test_refusals():
    a = torch.zeros((4096,), device="cuda")
    for args, status in [((B.F32, 1, 64, 8, 48, a, a, a, None, a, B.F32, 0, a), -2), ((B.F32, 0, 64, 8, 32, a, a, a, None, a, B.F32, 0, a), -2),
                         ((B.F32, 1, 0, 8, 32, a, a, a, None, a, B.F32, 0, a), -2), ((5, 1, 64, 8, 32, a, a, a, None, a, B.F32, 0, a), -3),
                         ((B.F32, 1, 64, 8, 32, a, a, a, None, a, 9, 0, a), -3), ((B.F32, 1, 64, 8, 32, None, a, a, None, a, B.F32, 0, a), -1),
                         ((B.F32, 1, 64, 8, 32, a, a, a[1:], None, a, B.F32, 0, a), -4),
                         ((B.BF16, 100, 4096, 1000, 32, a, a, a, None, a, B.F32, 0, None), -5)]:
        with pytest.raises(B.VggError) as e:
            B.vgg_fc_w4(*args)
        assert e.value.status == status, args
    with pytest.raises(B.VggError):
        B.vgg_fc_w4_quantize(64, 8, 31, a, a, a)
    with pytest.raises(B.VggError):
        B.vgg_fc_w4_dequantize(64, 0, 32, a, a, a)


def test_product_in_a_graph_and_on_another_stream():
    g = torch.Generator(device="cuda").manual_seed(1)
    In, Out, N, group = 1024, 200, 70, 64
    codes = torch.randint(0, 256, (Out, In // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.rand((Out, In // group), generator=g, device="cuda").to(torch.bfloat16)
    a = torch.randn((N, In), generator=g, device="cuda").to(torch.bfloat16)
    z, y = (torch.zeros((N, Out), device="cuda") for _ in range(2))
    ws = ws_bytes(B.vgg_fc_w4_workspace_bytes(B.BF16, N, In, Out, group))
    call = lambda out: B.vgg_fc_w4(B.BF16, N, In, Out, group, a, codes, scales, None, out, B.F32, 1, ws)  # noqa: E731
    call(z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(y)
    torch.cuda.synchronize()
    assert torch.equal(z, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y)
    for k in range(3):
        a.copy_(torch.randn((N, In), generator=g, device="cuda").to(torch.bfloat16))
        call(z)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, y), k


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shape", list(W4_TILES))
def test_product_by_every_tile_of_rows_and_outputs(shape, group):
    dtype, N, In, Out = shape
    g = torch.Generator(device="cuda").manual_seed(N + In)
    codes = torch.randint(0, 256, (Out, -(-In // 32) * 16), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((Out, -(-In // group)), generator=g, device="cuda") * 0.02 + 1e-3).to(torch.bfloat16)
    a = torch.randn((N, In), generator=g, device="cuda").to(TDT[dtype])
    b = torch.randn((Out,), generator=g, device="cuda")
    relu, zdt = group == 64, dtype if group == 32 else B.F32
    z = torch.full((N, Out), float("nan"), dtype=TDT[zdt], device="cuda")
    ws = ws_bytes(B.vgg_fc_w4_workspace_bytes(dtype, N, In, Out, group))
    ws.fill_(0xFF)
    B.vgg_fc_w4(dtype, N, In, Out, group, a, codes, scales, b, z, zdt, relu, ws)
    table, a64 = torch.from_numpy(np.concatenate((GRID, -GRID))).cuda(), a.double()
    for o in range(0, Out, 512):                                       # (the weights in 64 bits, some outputs at a time)
        c = codes[o : o + 512]
        w = table[torch.stack((c & 15, c >> 4), 2).flatten(1)[:, :In].int()]
        w *= scales[o : o + 512].double().repeat_interleave(group, 1)[:, :In]
        wt = w.t().contiguous()
        want, size = a64 @ wt + b[o : o + 512].double(), a64.abs() @ wt.abs() + b[o : o + 512].double().abs()
        check(z[:, o : o + 512].double(), want.clamp_min(0) if relu else want, size, zdt)
