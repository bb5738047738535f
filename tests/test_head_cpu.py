"""Host-only checks of the dense head: the workspace that it allocates covers every batch that it takes, and the tensors of a
call are looked at before anything is launched."""
from types import SimpleNamespace

import pytest
import torch

from paper_1810_09868_amd import binding as B
from paper_1810_09868_amd.head import DenseHead, workspace_bytes


@pytest.mark.parametrize("dtype,N,dims", [(B.BF16, 513, [128, 10000]), (B.BF16, 257, [168, 10755]), (B.BF16, 2000, [64, 64, 256, 5000]),
                                          (B.F32, 1000, [8, 64, 4096, 1000]), (B.F32, 1500, [24, 9000]), (B.F32, 130, [96, 64, 40, 10])])
def test_the_workspace_covers_every_number_of_rows(dtype, N, dims):
    # fewer rows are cut into more parts, so that no call's need grows with them throughout
    group, top = 64, 5
    have = workspace_bytes(dtype, N, dims, group, top)
    for i, o in zip(dims[:-1], dims[1:]):
        assert B.vgg_muon_workspace_bytes(dtype, 1, o, i) <= have
        for n in range(1, N + 1):
            for need in (B.vgg_fc_workspace_bytes(dtype, n, i, o), B.vgg_fc_bwd_workspace_bytes(dtype, n, i, o),
                         B.vgg_fc_w4_workspace_bytes(dtype, n, i, o, group)):
                assert need <= have, (n, i, o)
    for n in range(1, N + 1):
        assert max(B.vgg_log_probs_workspace_bytes(B.F32, n, dims[-1], t) for t in (0, top)) <= have, n


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_tensors_that_the_kernels_would_misread_are_refused(dtype):
    td, other = (torch.float32, torch.bfloat16) if dtype == B.F32 else (torch.bfloat16, torch.float32)
    head = SimpleNamespace(dtype=dtype, N=8, dims=[16, 8, 3], ws=torch.zeros(1))
    x, y = torch.zeros((4, 16), dtype=td), torch.zeros((4,), dtype=torch.int32)
    assert DenseHead._rows(head, x, y) == DenseHead._rows(head, x, None) == 4
    wrong_x = [x.to(other), x.to("meta"), x[0], x[:, :15], x.t().contiguous().t(), torch.zeros((9, 16), dtype=td), x[:0], x.double()]
    wrong_y = [y.long(), y.to("meta"), y[:3], y[:, None], torch.zeros((8,), dtype=torch.int32)[::2], y.float()]
    for a, b in [(a, y) for a in wrong_x] + [(x, b) for b in wrong_y]:
        with pytest.raises(ValueError):
            DenseHead._rows(head, a, b)
