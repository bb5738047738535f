"""A trained head with layer norms, put into another head: the same answers."""
import numpy as np
import pytest
import torch

from paper_1810_09868_amd import binding as B
from paper_1810_09868_amd.head import DenseHead

from test_gpu_head import DIMS
from test_gpu_head_training import batch, loaded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("mode", [dict(norm=True), dict(norm=True, dropout=0.25, pieces=True)])
def test_a_loaded_head_answers_as_the_trained_one(dtype, mode):
    head, _ = loaded(dtype, 40, mode, bias_lr=0.5)
    rng = np.random.default_rng(6)
    x, y = (torch.from_numpy(a).cuda() for a in batch(rng, 40))
    x = x.to(torch.bfloat16 if dtype == B.BF16 else torch.float32)
    for _ in range(3):
        head.train_step(x, y)
    other = DenseHead(dtype, 40, DIMS, **mode)
    other.load(head.w, head.b, head.gamma, head.beta)
    want, got = head.answer(x, y), other.answer(x, y)
    assert torch.equal(got.logp, want.logp) and torch.equal(got.top_idx, want.top_idx)
    other.load(head.w, head.b)
    assert not torch.equal(other.answer(x, y).logp, want.logp)
