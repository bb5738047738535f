"""The dense head with layer norm, dropout and a loss in pieces, run together: training steps against the same steps in 64 bits, what is
dropped anew in every step, a recorded step, answers after training."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_1810_09868_amd import binding as B
from paper_1810_09868_amd.head import DenseHead

from test_gpu_head import DIMS, ns64, parameters
from test_gpu_norm import EPS, kept, scale

pytestmark = pytest.mark.gpu

MODES = [dict(norm=True), dict(dropout=0.25), dict(pieces=True), dict(norm=True, dropout=0.5, pieces=True), dict(dropout=0.5, pieces=True)]


class Head64:
    def __init__(self, w, b, norm=False, dropout=0.0, pieces=False, seed=0):
        self.w, self.b = [a.astype(np.float64) for a in w], [a.astype(np.float64) for a in b]
        self.mom = [np.zeros_like(a) for a in self.w]
        self.norm, self.p, self.seed, self.steps = norm, dropout, seed, 0
        self.gamma, self.beta = [np.ones(a.shape[1]) for a in self.w], [np.zeros(a.shape[1]) for a in self.w]

    def gradients(self, x, y):
        n, last, a = len(y), len(self.w) - 1, x
        saved = []
        for l, w in enumerate(self.w):
            f = kept(n, w.shape[1], self.p, self.seed, self.steps, l) * scale(self.p) if self.p and l else np.ones(())
            xh = rstd = None
            h = a
            if self.norm:
                d = a - a.mean(1, keepdims=True)
                rstd = 1 / np.sqrt((d * d).mean(1, keepdims=True) + EPS)
                xh = d * rstd
                h = xh * self.gamma[l] + self.beta[l]
            h = h * f
            saved.append((a, h, f, xh, rstd))
            z = h @ w.T + self.b[l]
            a = np.maximum(z, 0) if l < last else z
        z = a - a.max(1, keepdims=True)
        lp = z - np.log(np.exp(z).sum(1, keepdims=True))
        dz = (np.exp(lp) - np.eye(lp.shape[1])[y]) / n
        out = {"w": [], "b": [], "gamma": [], "beta": []}
        for l in reversed(range(last + 1)):
            a, h, f, xh, rstd = saved[l]
            out["w"].insert(0, dz.T @ h)
            out["b"].insert(0, dz.sum(0))
            g = (dz @ self.w[l]) * f
            if self.norm:
                out["gamma"].insert(0, (g * xh).sum(0))
                out["beta"].insert(0, g.sum(0))
                g = g * self.gamma[l]
                g = rstd * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
            dz = g * (a > 0)
        return lp[np.arange(n), y], out

    def step(self, x, y, lr, mu, bias_lr):
        logp, g = self.gradients(x, y)
        for l, gw in enumerate(g["w"]):
            self.mom[l] = mu * self.mom[l] + gw
            self.w[l] = self.w[l] - lr * np.sqrt(max(1, gw.shape[0] / gw.shape[1])) * ns64(gw + mu * self.mom[l])
            self.b[l] = self.b[l] - bias_lr * g["b"][l]
            if self.norm:
                self.gamma[l] = self.gamma[l] - bias_lr * g["gamma"][l]
                self.beta[l] = self.beta[l] - bias_lr * g["beta"][l]
        self.steps += 1
        return logp


def loaded(dtype, N, mode, **more):
    w, b = parameters(0)
    head = DenseHead(dtype, N, DIMS, seed=99, **mode, **more)
    head.load([torch.from_numpy(a) for a in w], [torch.from_numpy(a) for a in b])
    return head, Head64(w, b, seed=99, **mode)


def batch(rng, n):
    return np.maximum(rng.standard_normal((n, DIMS[0])), 0).astype(np.float32), rng.integers(0, DIMS[-1], n).astype(np.int32)


@pytest.mark.parametrize("mode", MODES)
def test_steps_in_fp32_follow_64_bits(mode):
    head, ref = loaded(B.F32, 50, mode, lr=0.05, mu=0.9, bias_lr=0.1)
    rng = np.random.default_rng(1)
    for n in (50, 17, 1):
        x, y = batch(rng, n)
        logp = head.train_step(torch.from_numpy(x).cuda(), torch.from_numpy(y).cuda())
        want = ref.step(x.astype(np.float64), y, 0.05, 0.9, 0.1)
        # fp32 layers are 1e-6 off and a step (of 0.05 to a weight) 3e-5 of itself; three of them
        assert np.abs(logp.double().cpu().numpy() - want).max() < 1e-4
    pairs = list(zip(head.w + head.b, ref.w + ref.b)) + (list(zip(head.gamma + head.beta, ref.gamma + ref.beta)) if head.norm else [])
    for mine, other in pairs:
        assert np.linalg.norm(mine.double().cpu().numpy() - other) <= 2e-4 * np.linalg.norm(other)
    assert int(head.rng[1]) == (3 if head.dropout else 0)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("mode", MODES)
def test_gradients(dtype, mode):
    head, ref = loaded(dtype, 50, mode)
    td = torch.bfloat16 if dtype == B.BF16 else torch.float32
    x, y = batch(np.random.default_rng(2), 50)
    xt = torch.from_numpy(x).cuda().to(td)
    ref.w = [a.to(td).double().numpy() for a in map(torch.from_numpy, ref.w)]       # what the products read
    _, want = ref.gradients(xt.double().cpu().numpy(), y)
    head.train_step(xt, torch.from_numpy(y).cuda())
    # fp32: some 1e-6.  bf16: a layer's inputs are off by 1.1e-3 of themselves in the root mean square (2^-9 at most), its pre-activations by as much
    # of their width s, so that a ReLU decides otherwise with the probability 0.8 x 1.1e-3 s x density 0.4 / s = 3.5e-4, twice that in the second
    # layer: of 50 x 64 and 50 x 40 units 1.1 + 1.4 are expected, 8 at most in 999 of 1000.  Each moves a gradient by one of its 1000 to 1600 active terms, of
    # up to 1.5 times the common size: sqrt(8 / 1000) x 1.5 = 0.13; the roundings by themselves 0.01.
    limit = 0.13 if dtype == B.BF16 else 1e-5
    for mine, other in zip(head.dw + head.db + head.dgamma + head.dbeta, want["w"] + want["b"] + want["gamma"] + want["beta"]):
        assert np.linalg.norm(mine.double().cpu().numpy() - other) <= limit * np.linalg.norm(other)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("mode", MODES[3:])
def test_a_recorded_step_drops_anew(dtype, mode):
    td = torch.bfloat16 if dtype == B.BF16 else torch.float32
    eager, _ = loaded(dtype, 40, mode)
    graphed, _ = loaded(dtype, 40, mode)
    rng = np.random.default_rng(3)
    x, y = (torch.from_numpy(a).cuda() for a in batch(rng, 40))
    x = x.to(td)
    for h in (eager, graphed):
        h.train_step(x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.train_step(x, y)
    for _ in range(3):
        new = batch(rng, 40)
        x.copy_(torch.from_numpy(new[0]).cuda().to(td))
        y.copy_(torch.from_numpy(new[1]).cuda())
        want = eager.train_step(x, y).clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(graphed.logp[:40], want)
        assert all(torch.equal(a, b) for a, b in zip(eager.w + eager.b + eager.gamma + eager.beta, graphed.w + graphed.b + graphed.gamma + graphed.beta))
        assert int(graphed.rng[1]) == int(eager.rng[1])


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("mode", MODES)
def test_answers_are_of_the_same_layers(dtype, mode):
    td = torch.bfloat16 if dtype == B.BF16 else torch.float32
    head, _ = loaded(dtype, 64, mode, group=32, top=3)
    rng = np.random.default_rng(4)
    x, y = (torch.from_numpy(a).cuda() for a in batch(rng, 64))
    x = x.to(td)
    head.train_step(x, y)
    full = head.answer(x, y)
    a = x.double()
    for l, w in enumerate(head.operand):
        if head.norm:
            d = a - a.mean(1, keepdim=True)
            a = d / (d.square().mean(1, keepdim=True) + EPS).sqrt() * head.gamma[l].double() + head.beta[l].double()
        a = a @ w.double().t() + head.b[l].double()
        a = a.clamp_min(0) if l + 1 < len(head.w) else a
    lp = torch.log_softmax(a, 1)
    # (bf16: four tensors rounded to 2^-9 on the way to scores of some units; nothing is dropped)
    assert float((full.logp.double() - lp.gather(1, y.long()[:, None])[:, 0]).abs().max()) < (0.15 if dtype == B.BF16 else 1e-4)
    again = head.answer(x, y)
    assert torch.equal(full.logp, again.logp)
    head.quantize()
    few = head.answer(x, y)
    assert torch.isfinite(few.logp).all() and few.top_idx.shape == (64, 3)


def test_refusals():
    for wrong in (dict(dropout=1.0), dict(dropout=-0.1), dict(eps=0.0)):
        with pytest.raises(ValueError):
            DenseHead(B.F32, 4, [8, 3], **wrong)
    head = DenseHead(B.F32, 4, [8, 3], pieces=True)
    with pytest.raises(ValueError):
        head.train_step(torch.zeros((2, 8), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), 0.1)


def test_example_runs():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "train_and_serve_head.py"), "--steps", "21", "--norm", "--dropout", "0.1", "--pieces"],
                       capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "4-bit weights" in r.stdout and "one row" in r.stdout
