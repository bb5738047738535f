#!/usr/bin/env python3
"""Trains a classifier of dense layers on features, rounds it to 4 bits and lets it answer.

  python examples/train_and_serve_head.py [--dtype bf16|f32] [--steps 60] [--norm] [--dropout 0.1] [--pieces]

The features stand for a network's last pooled layer: 64 classes, each a direction of its own under noise and a ReLU.
Every weight matrix takes orthogonalised steps; the trained head then answers with the most likely classes, their log
probabilities and the entropy, from its fp32 or bf16 weights and from 4-bit ones.  --norm puts a layer norm in front of
every layer, --dropout drops a share of what goes between them, --pieces takes the loss without keeping the scores.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1810_09868_amd import binding as B  # noqa: E402
from paper_1810_09868_amd.head import DenseHead  # noqa: E402

FEATURES, HIDDEN, CLASSES, BATCH = 512, 256, 64, 100


def examples(n, centres, g):
    y = torch.randint(0, CLASSES, (n,), generator=g, device="cuda", dtype=torch.int32)
    x = (centres[y.long()] + 1.5 * torch.randn((n, FEATURES), generator=g, device="cuda")).clamp_min(0)
    return x, y


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--norm", action="store_true")
    ap.add_argument("--dropout", type=float, default=0.0)
    ap.add_argument("--pieces", action="store_true")
    a = ap.parse_args()
    dtype, td = (B.BF16, torch.bfloat16) if a.dtype == "bf16" else (B.F32, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(0)
    dims = [FEATURES, HIDDEN, HIDDEN, CLASSES]
    head = DenseHead(dtype, BATCH, dims, lr=0.02, norm=a.norm, dropout=a.dropout, pieces=a.pieces)
    head.load([torch.randn((o, i), generator=g, device="cuda") * (2.0 / i) ** 0.5 for i, o in zip(dims[:-1], dims[1:])],
              [torch.zeros(o, device="cuda") for o in dims[1:]])
    centres = torch.randn((CLASSES, FEATURES), generator=g, device="cuda")
    for step in range(a.steps):
        x, y = examples(BATCH, centres, g)
        logp = head.train_step(x.to(td), y)
        if step % 20 == 0 or step + 1 == a.steps:
            print("step %3d: mean log probability of the label %.4f" % (step, float(logp.mean())))
    x, y = examples(BATCH, centres, g)
    for name in (a.dtype, "4-bit"):
        size = head.quantize() if name == "4-bit" else sum(w.numel() * w.element_size() for w in head.operand)
        r = head.answer(x.to(td), y)
        print("%5s weights, %7d bytes: %5.1f %% right, mean log probability %.4f, entropy %.4f" % (
            name, size, 100 * float((r.top_idx[:, 0] == y).float().mean()), float(r.logp.mean()), float(r.entropy.mean())))
    one = head.answer(x[:1].to(td))
    print("one row: " + ", ".join("class %d %.3f" % (int(k), float(v.exp())) for k, v in zip(one.top_idx[0], one.top_logp[0])))


if __name__ == "__main__":
    main()
