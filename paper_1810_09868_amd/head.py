"""A classifier of dense layers: trained with orthogonalised updates, held in 4 bits, answering with log probabilities.

Buffer management around binding's entry points, as model.Vgg19 around the whole network's (no arithmetic: all compute
happens in libvgg_mi355x.so).  The layers are those of the network's classifier (dense, ReLU between) on features of any
width; weights [Out][In] and biases are fp32, activations `dtype`.
"""
from __future__ import annotations

from typing import List, NamedTuple, Optional, Sequence

import torch

from . import binding as B


class Answer(NamedTuple):
    """Views of the head's buffers, overwritten by its next call (top_*: none where no alternatives were asked for)."""
    logp: Optional[torch.Tensor]      # [N] of the given labels
    entropy: torch.Tensor             # [N]
    top_logp: Optional[torch.Tensor]  # [N][top]
    top_idx: Optional[torch.Tensor]   # [N][top] int32


def _bytes(n: int) -> torch.Tensor:
    return torch.empty((max(int(n), 16),), dtype=torch.uint8, device="cuda")


def workspace_bytes(dtype: int, N: int, dims: Sequence[int], group: int, top: int) -> int:
    """What the calls of a head of these layers need at most, over every number of rows up to N: fewer rows may need more, since
    they are cut into more parts."""
    need = [B.vgg_muon_workspace_bytes(d, 1, o, i) for d in (B.F32, B.BF16) for i, o in zip(dims[:-1], dims[1:])]
    for n in range(1, N + 1):
        need += [B.vgg_log_probs_workspace_bytes(B.F32, n, dims[-1], t) for t in (0, top)]
        for i, o in zip(dims[:-1], dims[1:]):
            need += [B.vgg_fc_workspace_bytes(dtype, n, i, o), B.vgg_fc_bwd_workspace_bytes(dtype, n, i, o),
                     B.vgg_fc_w4_workspace_bytes(dtype, n, i, o, group)]
    return max(need)


class DenseHead:
    """`dims` are the layers' widths, features first and classes last; at most N rows a call.  `update_dtype`: how exact the
    products of the updates are (vgg_muon_update; BF16: operands of 11 bits), whatever `dtype` the layers have."""

    def __init__(self, dtype: int, N: int, dims: Sequence[int], lr: float = 0.02, mu: float = 0.95, weight_decay: float = 0.0,
                 bias_lr: float = 0.01, ns_steps: int = 5, group: int = 64, top: int = 5, update_dtype: int = B.F32):
        if not torch.cuda.is_available():
            raise RuntimeError("DenseHead needs a GPU: the HIP library is the only implementation")
        if len(dims) < 2 or N < 1:
            raise ValueError("a head has at least one layer and one row")
        if dtype not in (B.F32, B.BF16) or update_dtype not in (B.F32, B.BF16) or group not in (32, 64, 128) or not 0 <= top <= B.MAX_TOP:
            raise ValueError("dtypes are F32 or BF16, group 32, 64 or 128, top 0 to %d" % B.MAX_TOP)
        if dtype == B.BF16 and any(d % 8 for d in dims[:-1]):
            raise ValueError("bf16: layer inputs are multiples of 8 (vgg_fc_bwd)")
        self.dtype, self.N, self.dims, self.group, self.top = dtype, N, list(dims), group, min(top, dims[-1])
        self.update_dtype = update_dtype
        self.lr, self.mu, self.weight_decay, self.bias_lr, self.ns_steps = lr, mu, weight_decay, bias_lr, ns_steps
        td = torch.bfloat16 if dtype == B.BF16 else torch.float32
        f32 = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        pairs = list(zip(dims[:-1], dims[1:]))
        self.w, self.b = [f32(o, i) for i, o in pairs], [f32(o) for _, o in pairs]
        self.momentum = [f32(o, i) for i, o in pairs]
        # what the products read: the weights themselves, or their bf16 copies
        self.operand = self.w if dtype == B.F32 else [torch.zeros((o, i), dtype=td, device="cuda") for i, o in pairs]
        self.act = [torch.empty((N, o), dtype=td, device="cuda") for _, o in pairs[:-1]]
        self.logits, self.dz = f32(N, dims[-1]), [f32(N, o) for _, o in pairs]
        self.dw, self.db = [f32(o, i) for i, o in pairs], [f32(o) for _, o in pairs]
        self.logp, self.entropy, self.stats = f32(N), f32(N), f32(N, 2)
        self.g_logp, self.g_entropy = f32(N), f32(N)
        self.top_logp, self.top_idx = f32(N, self.top), torch.zeros((N, self.top), dtype=torch.int32, device="cuda")
        self.codes: List[torch.Tensor] = []
        self.scales: List[torch.Tensor] = []
        self.ws = _bytes(workspace_bytes(dtype, N, dims, group, self.top))

    def load(self, weights: Sequence[torch.Tensor], biases: Sequence[torch.Tensor]) -> None:
        """Takes fp32 parameters; momentum starts from zero, and 4-bit weights of earlier ones are dropped."""
        if [tuple(t.shape) for t in weights] != [tuple(w.shape) for w in self.w] or [tuple(t.shape) for t in biases] != [tuple(b.shape) for b in self.b]:
            raise ValueError("a weight [out][in] and a bias [out] for each layer of %s" % self.dims)
        for mine, given in zip(self.w + self.b, list(weights) + list(biases)):
            mine.copy_(given)
        for m in self.momentum:
            m.zero_()
        self.codes, self.scales = [], []
        self._refresh()

    def _refresh(self) -> None:
        if self.dtype == B.BF16:
            for w, c in zip(self.w, self.operand):
                B.vgg_convert(B.F32, B.BF16, w.numel(), w, c)

    def _rows(self, x: torch.Tensor, labels: Optional[torch.Tensor]) -> int:
        """The number of rows of a call, whose tensors are what the kernels take them for."""
        td = torch.bfloat16 if self.dtype == B.BF16 else torch.float32
        if x.dim() != 2 or not 1 <= x.shape[0] <= self.N or x.shape[1] != self.dims[0] or x.dtype != td or x.device != self.ws.device or not x.is_contiguous():
            raise ValueError("features are contiguous [1..%d][%d], %s on %s" % (self.N, self.dims[0], td, self.ws.device))
        n = x.shape[0]
        if labels is not None and (labels.shape != (n,) or labels.dtype != torch.int32 or labels.device != x.device or not labels.is_contiguous()):
            raise ValueError("labels are contiguous [%d], int32 on %s" % (n, x.device))
        return n

    def _forward(self, x: torch.Tensor, n: int) -> None:
        a, last = x, len(self.w) - 1
        for l, w in enumerate(self.operand):
            o, i = w.shape
            z = self.logits if l == last else self.act[l]
            B.vgg_fc(self.dtype, n, i, o, a, w, self.b[l], z, B.F32 if l == last else self.dtype, l < last, self.ws)
            a = z

    def train_step(self, x: torch.Tensor, labels: torch.Tensor, entropy_weight: float = 0.0) -> torch.Tensor:
        """One step on features x [n][dims[0]] and int32 labels: the mean of -log p[label] - entropy_weight * entropy is
        decreased; every weight matrix takes an orthogonalised step, biases a plain one.  Returns the rows' log probabilities
        before the step (a view)."""
        if labels is None:
            raise ValueError("a training step needs labels")
        n, K = self._rows(x, labels), self.dims[-1]
        self._forward(x, n)
        B.vgg_log_probs(B.F32, n, K, self.logits, labels, 0, self.logp, self.entropy, None, None, self.stats, self.ws)
        self.g_logp[:n].fill_(-1.0 / n)
        self.g_entropy[:n].fill_(-entropy_weight / n)
        B.vgg_log_probs_bwd(B.F32, n, K, self.logits, labels, self.stats, self.entropy, self.g_logp, self.g_entropy if entropy_weight else None,
                            self.dz[-1])
        for l in reversed(range(len(self.w))):
            o, i = self.w[l].shape
            B.vgg_fc_bwd(self.dtype, n, i, o, self.act[l - 1] if l else x, self.operand[l], self.dz[l], self.dw[l], self.db[l],
                         self.dz[l - 1] if l else None, l > 0, self.ws)
        for l, w in enumerate(self.w):
            B.vgg_muon_update(self.update_dtype, 1, *w.shape, self.ns_steps, w, self.dw[l], self.momentum[l], self.lr, self.mu, True,
                              self.weight_decay, self.ws)
            B.vgg_sgd_update(self.b[l].numel(), self.b[l], self.db[l], self.bias_lr)
        self.codes, self.scales = [], []
        self._refresh()
        return self.logp[:n]

    def quantize(self) -> int:
        """Rounds the weights as they are to 4 bits; answers are from these until the next training step.  Returns their bytes."""
        self.codes, self.scales = [], []
        for w in self.w:
            o, i = w.shape
            c = torch.empty((o, -(-i // 32) * 16), dtype=torch.uint8, device="cuda")
            s = torch.empty((o, -(-i // self.group)), dtype=torch.bfloat16, device="cuda")
            B.vgg_fc_w4_quantize(i, o, self.group, w, c, s)
            self.codes.append(c)
            self.scales.append(s)
        return sum(c.numel() + 2 * s.numel() for c, s in zip(self.codes, self.scales))

    def answer(self, x: torch.Tensor, labels: Optional[torch.Tensor] = None) -> Answer:
        """Log probabilities of the given labels, entropy and the most likely classes of features x [n][dims[0]]."""
        n, last, a = self._rows(x, labels), len(self.w) - 1, x
        if not self.codes:
            self._forward(x, n)
        else:
            for l, (c, s) in enumerate(zip(self.codes, self.scales)):
                o, i = self.w[l].shape
                z = self.logits if l == last else self.act[l]
                B.vgg_fc_w4(self.dtype, n, i, o, self.group, a, c, s, self.b[l], z, B.F32 if l == last else self.dtype, l < last,
                            self.ws)
                a = z
        B.vgg_log_probs(B.F32, n, self.dims[-1], self.logits, labels, self.top, self.logp if labels is not None else None,
                        self.entropy, self.top_logp if self.top else None, self.top_idx if self.top else None, None, self.ws)
        return Answer(self.logp[:n] if labels is not None else None, self.entropy[:n], self.top_logp[:n] if self.top else None,
                      self.top_idx[:n] if self.top else None)
