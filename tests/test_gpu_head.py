"""The dense head: training step, rounding and answers run together, against the same steps in 64 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_1810_09868_amd import binding as B
from paper_1810_09868_amd.head import DenseHead

pytestmark = pytest.mark.gpu

DIMS = [96, 64, 40, 10]


def parameters(seed):
    rng = np.random.default_rng(seed)
    w = [(rng.standard_normal((o, i)) * np.sqrt(2.0 / i)).astype(np.float32) for i, o in zip(DIMS[:-1], DIMS[1:])]
    return w, [(0.1 * rng.standard_normal(o)).astype(np.float32) for o in DIMS[1:]]


def ns64(u):
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (np.sqrt((x * x).sum()) + 1e-7)
    for _ in range(5):
        g = x @ x.T
        x = 3.4445 * x + (-4.775 * g + 2.0315 * (g @ g)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def step64(w, b, mom, x, y, lr, mu, bias_lr, weight):
    acts = [x]
    for l in range(len(w)):
        z = acts[-1] @ w[l].T + b[l]
        acts.append(np.maximum(z, 0) if l + 1 < len(w) else z)
    z = acts[-1] - acts[-1].max(1, keepdims=True)
    lp = z - np.log(np.exp(z).sum(1, keepdims=True))
    p, n = np.exp(lp), len(y)
    H = -(p * lp).sum(1, keepdims=True)
    dz = (p - np.eye(p.shape[1])[y]) / n + weight / n * p * (lp + H)
    grads = []
    for l in reversed(range(len(w))):
        grads.insert(0, (dz.T @ acts[l], dz.sum(0)))
        if l:
            dz = (dz @ w[l]) * (acts[l] > 0)
    for l, (gw, gb) in enumerate(grads):
        mom[l] = mu * mom[l] + gw
        w[l] = w[l] - lr * np.sqrt(max(1, w[l].shape[0] / w[l].shape[1])) * ns64(gw + mu * mom[l])
        b[l] = b[l] - bias_lr * gb
    return lp[np.arange(n), y]


@pytest.mark.parametrize("weight", [0.0, 0.1])
def test_training_steps_in_fp32_follow_64_bits(weight):
    w, b = parameters(0)
    head = DenseHead(B.F32, 50, DIMS, lr=0.05, mu=0.9, bias_lr=0.1)
    head.load([torch.from_numpy(a) for a in w], [torch.from_numpy(a) for a in b])
    w, b = [a.astype(np.float64) for a in w], [a.astype(np.float64) for a in b]
    mom = [np.zeros_like(a) for a in w]
    rng = np.random.default_rng(1)
    for n in (50, 17, 1):
        x, y = np.maximum(rng.standard_normal((n, DIMS[0])), 0).astype(np.float32), rng.integers(0, DIMS[-1], n).astype(np.int32)
        logp = head.train_step(torch.from_numpy(x).cuda(), torch.from_numpy(y).cuda(), weight)
        want = step64(w, b, mom, x.astype(np.float64), y, 0.05, 0.9, 0.1, weight)
        # fp32 layers are 1e-6 off and a step (of 0.05 to a weight) 3e-5 of itself; three of them
        assert np.abs(logp.double().cpu().numpy() - want).max() < 1e-4
    for mine, ref in zip(head.w + head.b, w + b):
        assert np.linalg.norm(mine.double().cpu().numpy() - ref) <= 2e-4 * np.linalg.norm(ref)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_it_learns_and_its_four_bits_answer_alike(dtype):
    td = torch.bfloat16 if dtype == B.BF16 else torch.float32
    g = torch.Generator(device="cuda").manual_seed(2)
    w, b = parameters(3)
    head = DenseHead(dtype, 64, DIMS, lr=0.03, group=32, top=3)
    head.load([torch.from_numpy(a) for a in w], [torch.from_numpy(a) for a in b])
    centres = torch.randn((10, DIMS[0]), generator=g, device="cuda")

    def batch(n):
        y = torch.randint(0, 10, (n,), generator=g, device="cuda", dtype=torch.int32)
        return (centres[y.long()] + 0.5 * torch.randn((n, DIMS[0]), generator=g, device="cuda")).clamp_min(0).to(td), y

    first = float(head.train_step(*batch(64)).mean())
    for _ in range(40):
        last = float(head.train_step(*batch(64)).mean())
    assert last > -0.1 > first
    x, y = batch(64)
    full = head.answer(x, y)
    z = head.logits.double().clone()
    assert (full.top_idx[:, 0] == y).float().mean() > 0.95
    lp = torch.log_softmax(z, 1)
    assert float((full.logp.double() - lp.gather(1, y.long()[:, None])[:, 0]).abs().max()) < 1e-5
    assert float((full.entropy.double() + (lp.exp() * lp).sum(1)).abs().max()) < 1e-5
    assert head.quantize() < sum(p.numel() for p in head.w)            # bytes of 4-bit weights and their scales
    few = head.answer(x, y)
    assert (few.top_idx[:, 0] == y).float().mean() > 0.95
    one = head.answer(x[5:6].contiguous())
    assert one.logp is None and int(one.top_idx[0, 0]) == int(few.top_idx[5, 0]) and one.top_logp.shape == (1, 3)


def test_refusals():
    head = DenseHead(B.F32, 4, [8, 3])
    with pytest.raises(ValueError):
        head.answer(torch.zeros((5, 8), device="cuda"))
    with pytest.raises(ValueError):
        head.answer(torch.zeros((2, 9), device="cuda"))
    with pytest.raises(ValueError):
        DenseHead(B.BF16, 4, [9, 3])
    with pytest.raises(ValueError):
        DenseHead(B.F32, 4, [9])


def test_example_runs():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "train_and_serve_head.py"), "--steps", "21"], capture_output=True,
                       text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "4-bit weights" in r.stdout and "one row" in r.stdout


def ns_gpu(u):
    x = u.t().contiguous() if u.shape[0] > u.shape[1] else u
    x = x / (torch.linalg.vector_norm(x) + 1e-7)
    for _ in range(5):
        g = x @ x.t().contiguous()
        x = 3.4445 * x + (-4.775 * g + 2.0315 * (g @ g)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


@pytest.mark.parametrize("dims,rows", [([200, 300, 5000], (640, 100, 3)), ([8, 64, 4096, 1000], (1000, 640, 128, 41))])
def test_wide_heads_follow_64_bits_at_any_number_of_rows(dims, rows):
    # rows in parts, updates by product tiles, every plan of the dense backward, batches that need more workspace than the largest.
    # The change of the weights: Newton-Schulz is 3e-5 off, and enlarges a gradient's rounding (1e-6) up to 485-fold: 1e-3 in all.
    # A step changes a score by less than 1, of which 5e-4 are as far as the log probabilities are off.
    g = torch.Generator(device="cuda").manual_seed(7)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    w = [normal(o, i) * (2.0 / i) ** 0.5 for i, o in zip(dims[:-1], dims[1:])]
    b = [0.1 * normal(o) for o in dims[1:]]
    lr, mu, bias_lr, weight = 0.01, 0.9, 0.1, 0.05
    head = DenseHead(B.F32, rows[0], dims, lr=lr, mu=mu, bias_lr=bias_lr)
    head.load(w, b)
    first = [a.double() for a in w]
    w, b = [a.double() for a in w], [a.double() for a in b]
    mom = [torch.zeros_like(a) for a in w]
    for n in rows:
        x, y = normal(n, dims[0]).clamp_min(0), torch.randint(0, dims[-1], (n,), generator=g, device="cuda", dtype=torch.int32)
        logp = head.train_step(x, y, weight)
        acts = [x.double()]
        for l in range(len(w)):
            z = acts[-1] @ w[l].t().contiguous() + b[l]
            acts.append(z.clamp_min(0) if l + 1 < len(w) else z)
        lp = torch.log_softmax(acts[-1], 1)
        p = lp.exp()
        dz = p / n + weight / n * p * (lp - (p * lp).sum(1, keepdim=True))
        dz[torch.arange(n, device="cuda"), y.long()] -= 1.0 / n
        assert float((logp.double() - lp.gather(1, y.long()[:, None])[:, 0]).abs().max()) < 5e-4
        for l in reversed(range(len(w))):
            gw, gb = dz.t().contiguous() @ acts[l], dz.sum(0)
            if l:
                dz = (dz @ w[l]) * (acts[l] > 0)
            mom[l] = mu * mom[l] + gw
            w[l] = w[l] - lr * max(1.0, w[l].shape[0] / w[l].shape[1]) ** 0.5 * ns_gpu(gw + mu * mom[l])
            b[l] = b[l] - bias_lr * gb
    for mine, ref, was in zip(head.w, w, first):
        assert float((mine.double() - ref).norm() / (ref - was).norm()) < 1e-3


@pytest.mark.parametrize("N,n,dims", [(513, 512, [128, 10000]), (257, 256, [168, 10755])])
def test_a_batch_that_needs_more_workspace_than_the_largest(N, n, dims):
    head = DenseHead(B.BF16, N, dims)
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn((dims[1], dims[0]), generator=g, device="cuda") * 0.1).to(torch.bfloat16)
    head.load([w.float()], [torch.zeros(dims[1], device="cuda")])
    x = torch.randn((n, dims[0]), generator=g, device="cuda").to(torch.bfloat16)
    y = torch.randint(0, dims[1], (n,), generator=g, device="cuda", dtype=torch.int32)
    logp = head.train_step(x, y)
    want = torch.log_softmax(x.double() @ w.double().t().contiguous(), 1)
    assert float((logp.double() - want.gather(1, y.long()[:, None])[:, 0]).abs().max()) < 1e-4


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_tensors_that_the_kernels_would_misread_are_refused(dtype):
    head = DenseHead(dtype, 8, [16, 8, 3])
    td, other = (torch.float32, torch.bfloat16) if dtype == B.F32 else (torch.bfloat16, torch.float32)
    x, y = torch.zeros((4, 16), dtype=td, device="cuda"), torch.zeros((4,), dtype=torch.int32, device="cuda")
    wrong_x = [x.to(other), x.cpu(), x[0], x[:, :15], x.t().contiguous().t(), torch.zeros((9, 16), dtype=td, device="cuda"), x[:0], x.double()]
    wrong_y = [y.long(), y.cpu(), y[:3], y[:, None], torch.zeros((8,), dtype=torch.int32, device="cuda")[::2], y.float()]
    for a, b in [(a, y) for a in wrong_x] + [(x, b) for b in wrong_y]:
        for call in (head.train_step, head.answer):
            with pytest.raises(ValueError):
                call(a, b)
    with pytest.raises(ValueError):
        head.train_step(x, None)
    w, b = [torch.zeros((8, 16)), torch.zeros((3, 8))], [torch.zeros(8), torch.zeros(3)]
    for ws, bs in ((w[:1], b), (w, b[:1]), ([w[0], torch.zeros((1, 8))], b), (w, [b[0], torch.zeros(1)])):
        with pytest.raises(ValueError):
            head.load(ws, bs)
    head.load(w, b)
    for bad in (dict(dtype=5), dict(group=16), dict(top=65), dict(top=-1)):
        with pytest.raises(ValueError):
            DenseHead(**{**dict(dtype=dtype, N=4, dims=[8, 3]), **bad})
    assert head.answer(x, y).logp.shape == (4,) and head.train_step(x, y).shape == (4,)


def test_minibatches_are_parts_of_longer_tensors():
    x = torch.randn((100, 16), device="cuda")
    y = torch.randint(0, 3, (100,), dtype=torch.int32, device="cuda")
    w, b = [torch.randn((8, 16)), torch.randn((3, 8))], [torch.randn(8), torch.randn(3)]
    got = []
    for copy in (False, True):
        head = DenseHead(B.F32, 50, [16, 8, 3])
        head.load(w, b)
        for first, last in ((0, 50), (50, 99), (1, 4), (99, 100)):
            part = y[first:last].clone() if copy else y[first:last]
            head.train_step(x[first:last], part, 0.1)
        got.append([t.clone() for t in head.w] + [head.answer(x[50:100], y[50:100].clone() if copy else y[50:100]).logp.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("update_dtype", [None, B.BF16])
def test_weights_meet_exact_updates_unless_short_operands_are_asked_for(update_dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    kw = {} if update_dtype is None else dict(update_dtype=update_dtype)
    head = DenseHead(B.BF16, 96, [256, 200, 120], lr=0.02, mu=0.9, weight_decay=0.01, **kw)
    head.load([torch.randn((o, i), generator=g, device="cuda") * (2.0 / i) ** 0.5 for i, o in ((256, 200), (200, 120))],
              [torch.zeros(200, device="cuda"), torch.zeros(120, device="cuda")])
    for _ in range(2):
        w, mom = [t.clone() for t in head.w], [t.clone() for t in head.momentum]
        x, y = torch.randn((96, 256), generator=g, device="cuda").to(torch.bfloat16), torch.randint(0, 120, (96,), device="cuda", dtype=torch.int32)
        head.train_step(x, y)
        for l, (theta, m) in enumerate(zip(w, mom)):
            shape, dt = (1, *theta.shape), B.F32 if update_dtype is None else update_dtype
            ws = torch.empty(B.vgg_muon_workspace_bytes(dt, *shape), dtype=torch.uint8, device="cuda")
            B.vgg_muon_update(dt, *shape, 5, theta, head.dw[l], m, 0.02, 0.9, True, 0.01, ws)
            assert torch.equal(theta, head.w[l]) and torch.equal(m, head.momentum[l])
