"""Host-only: what a head loads, layer norms among it (its buffers stand on the CPU here: loading computes nothing)."""
from types import SimpleNamespace

import pytest
import torch

from paper_1810_09868_amd import binding as B
from paper_1810_09868_amd.head import DenseHead

DIMS = [6, 5, 3]


def head(norm):
    pairs = list(zip(DIMS[:-1], DIMS[1:]))
    full = lambda *s: torch.full(s, 9.0)  # noqa: E731
    return SimpleNamespace(dims=DIMS, dtype=B.F32, norm=norm, w=[full(o, i) for i, o in pairs], b=[full(o) for _, o in pairs], momentum=[full(o, i) for i, o in pairs],
                           gamma=[full(i) for i, _ in pairs if norm], beta=[full(i) for i, _ in pairs if norm], rng=torch.tensor([5, 7]), codes=[1], scales=[1],
                           _refresh=lambda: None)


def given(gen):
    pairs = list(zip(DIMS[:-1], DIMS[1:]))
    draw = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    return [draw(o, i) for i, o in pairs], [draw(o) for _, o in pairs], [draw(i) for i, _ in pairs], [draw(i) for i, _ in pairs]


def test_layer_norms_are_loaded():
    w, b, gamma, beta = given(torch.Generator().manual_seed(1))
    h = head(True)
    DenseHead.load(h, w, b, gamma, beta)
    for mine, theirs in zip(h.w + h.b + h.gamma + h.beta, w + b + gamma + beta):
        assert torch.equal(mine, theirs) and mine is not theirs
    assert all((m == 0).all() for m in h.momentum) and h.rng.tolist() == [5, 0] and h.codes == h.scales == []
    DenseHead.load(h, w, b, beta=beta)                 # the other from where layer norms begin
    assert all((g == 1).all() for g in h.gamma) and all(torch.equal(*t) for t in zip(h.beta, beta))
    DenseHead.load(h, w, b, h.gamma, h.beta)           # a head's own
    assert all((g == 1).all() for g in h.gamma) and all(torch.equal(*t) for t in zip(h.beta, beta))
    DenseHead.load(h, w, b)
    assert all((g == 1).all() for g in h.gamma) and all((t == 0).all() for t in h.beta)
    plain = head(False)
    DenseHead.load(plain, w, b)
    assert torch.equal(plain.w[0], w[0])
    DenseHead.load(plain, w, b, [], [])                # what a head without layer norms has of them
    assert torch.equal(plain.w[1], w[1])


def test_layer_norms_that_do_not_fit_are_refused_before_anything_is_loaded():
    w, b, gamma, beta = given(torch.Generator().manual_seed(2))
    for h, more in ((head(True), (gamma[:1], beta)), (head(True), (gamma, [t[:2] for t in beta])), (head(True), ([], [])), (head(False), (gamma, beta)), (head(False), (None, beta))):
        with pytest.raises(ValueError):
            DenseHead.load(h, w, b, *more)
        assert all((t == 9).all() for t in h.w + h.b + h.gamma + h.beta + h.momentum)
