"""A classifier of dense layers: trained with orthogonalised updates, held in 4 bits, answering with log probabilities; with
layer norm in front of its layers, dropout between them and a loss that takes its scores in pieces, where they are asked for.

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


def workspace_bytes(dtype: int, N: int, dims: Sequence[int], group: int, top: int, norm: bool = False, pieces: bool = False) -> int:
    """What the calls of a head of these layers need at most, over every number of rows up to N: fewer rows may need more, since
    they are cut into more parts."""
    need = [B.vgg_muon_workspace_bytes(d, 1, o, i) for d in (B.F32, B.BF16) for i, o in zip(dims[:-1], dims[1:])]
    for n in range(1, N + 1):
        need += [B.vgg_log_probs_workspace_bytes(B.F32, n, dims[-1], t) for t in (0, top)]
        for i, o in zip(dims[:-1], dims[1:]):
            need += [B.vgg_fc_workspace_bytes(dtype, n, i, o), B.vgg_fc_bwd_workspace_bytes(dtype, n, i, o),
                     B.vgg_fc_w4_workspace_bytes(dtype, n, i, o, group)]
            if norm:
                need.append(B.vgg_layer_norm_bwd_workspace_bytes(dtype, B.F32, n, i))
        if pieces:
            need += [B.vgg_fc_xent_workspace_bytes(dtype, n, *dims[-2:]), B.vgg_fc_xent_bwd_workspace_bytes(dtype, n, *dims[-2:])]
    return max(need)


class DenseHead:
    """`dims` are the layers' widths, features first and classes last; at most N rows a call.  `update_dtype`: how exact the
    products of the updates are (vgg_muon_update; BF16: operands of 11 bits), whatever `dtype` the layers have.

    norm: every layer takes the layer norm of what comes to it, with a scale and a shift of its own, learned at bias_lr.
    dropout: the share of what leaves a hidden layer (norm: of its layer norm) that a training step drops, anew in each
    step, by `seed`.  pieces: a training step forms the classes' scores and their gradients in pieces (vgg_fc_xent), so that
    nothing of [N][classes] is kept where that is much; answers have them all."""

    def __init__(self, dtype: int, N: int, dims: Sequence[int], lr: float = 0.02, mu: float = 0.95, weight_decay: float = 0.0,
                 bias_lr: float = 0.01, ns_steps: int = 5, group: int = 64, top: int = 5, update_dtype: int = B.F32, norm: bool = False,
                 dropout: float = 0.0, pieces: bool = False, seed: int = 0, eps: float = 1e-5):
        if not torch.cuda.is_available():
            raise RuntimeError("DenseHead needs a GPU: the HIP library is the only implementation")
        if len(dims) < 2 or N < 1:
            raise ValueError("a head has at least one layer and one row")
        if dtype not in (B.F32, B.BF16) or update_dtype not in (B.F32, B.BF16) or group not in (32, 64, 128) or not 0 <= top <= B.MAX_TOP:
            raise ValueError("dtypes are F32 or BF16, group 32, 64 or 128, top 0 to %d" % B.MAX_TOP)
        if not 0 <= dropout < 1 or not eps > 0:
            raise ValueError("dropout from 0 to below 1, eps above 0")
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
        self.norm, self.dropout, self.pieces, self.eps = norm, float(dropout), pieces, eps
        self.gamma, self.beta = [torch.ones(i, device="cuda") for i, _ in pairs if norm], [f32(i) for i, _ in pairs if norm]
        self.normed = [torch.empty((N, i), dtype=td, device="cuda") for i, _ in pairs if norm]
        self.norm_stats = [f32(N, 2) for _ in pairs if norm]
        self.dgamma, self.dbeta = [f32(i) for i, _ in pairs if norm], [f32(i) for i, _ in pairs if norm]
        self.dx = f32(N, dims[0]) if norm else None
        self.rng = torch.tensor([seed, 0], dtype=torch.int64, device="cuda")     # seed and training step
        # (pieces: scores are there from the first answer on)
        self.logits = None if pieces else f32(N, dims[-1])
        self.dz = [f32(N, o) for _, o in (pairs[:-1] if pieces else pairs)]
        self.dw, self.db = [f32(o, i) for i, o in pairs], [f32(o) for _, o in pairs]
        self.logp, self.entropy, self.stats = f32(N), f32(N), f32(N, 2)
        self.g_logp, self.g_entropy = f32(N), f32(N)
        self.top_logp, self.top_idx = f32(N, self.top), torch.zeros((N, self.top), dtype=torch.int32, device="cuda")
        self.codes: List[torch.Tensor] = []
        self.scales: List[torch.Tensor] = []
        self.ws = _bytes(workspace_bytes(dtype, N, dims, group, self.top, norm, pieces))

    def load(self, weights: Sequence[torch.Tensor], biases: Sequence[torch.Tensor], gamma: Optional[Sequence[torch.Tensor]] = None,
             beta: Optional[Sequence[torch.Tensor]] = None) -> None:
        """Takes fp32 parameters; gamma and beta are the layer norms' scales and shifts, 1 and 0 where they are not given.  Momentum starts
        from zero, dropout from step 0, and 4-bit weights of earlier parameters are dropped."""
        shapes = lambda ts: [tuple(t.shape) for t in ts]  # noqa: E731
        if shapes(weights) != shapes(self.w) or shapes(biases) != shapes(self.b):
            raise ValueError("a weight [out][in] and a bias [out] for each layer of %s" % self.dims)
        if any(given is not None and shapes(given) != shapes(self.gamma) for given in (gamma, beta)):
            raise ValueError("a scale and a shift [in] for each layer of %s%s" % (self.dims, "" if self.norm else ", of a head with layer norms"))
        for mine, given in zip(self.w + self.b, list(weights) + list(biases)):
            mine.copy_(given)
        for own, given, start in ((self.gamma, gamma, 1.0), (self.beta, beta, 0.0)):
            for l, t in enumerate(own):
                t.fill_(start) if given is None else t.copy_(given[l])
        for t in self.momentum + [self.rng[1:]]:
            t.zero_()
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

    def _input(self, l: int, a: torch.Tensor, n: int, train: bool) -> torch.Tensor:
        """What layer l takes of what comes to it: its layer norm, without what this training step drops."""
        i, p = self.dims[l], self.dropout if train and l else 0.0
        if self.norm:
            B.vgg_layer_norm(self.dtype, n, i, a, self.gamma[l], self.beta[l], self.eps, p, self.rng, l, self.normed[l],
                             self.norm_stats[l] if train else None)
            return self.normed[l]
        if p:
            B.vgg_dropout(self.dtype, n, i, a, p, self.rng, l, a)      # (in place: a ReLU's output, whose zeros stay what they are)
        return a

    def _forward(self, x: torch.Tensor, n: int, train: bool = False) -> List[torch.Tensor]:
        """The layers' inputs; scores are in logits, but where a training step takes them in pieces."""
        a, last, inputs = x, len(self.w) - 1, []
        for l, w in enumerate(self.operand):
            o, i = w.shape
            inputs.append(self._input(l, a, n, train))
            if l == last and train and self.pieces:
                break
            z = self._scores() if l == last else self.act[l]
            B.vgg_fc(self.dtype, n, i, o, inputs[l], w, self.b[l], z, B.F32 if l == last else self.dtype, l < last, self.ws)
            a = z
        return inputs

    def _scores(self) -> torch.Tensor:
        if self.logits is None:
            self.logits = torch.zeros((self.N, self.dims[-1]), device="cuda")
        return self.logits

    def train_step(self, x: torch.Tensor, labels: torch.Tensor, entropy_weight: float = 0.0) -> torch.Tensor:
        """One step on features x [n][dims[0]] and int32 labels: the mean of -log p[label] - entropy_weight * entropy is
        decreased; every weight matrix takes an orthogonalised step, biases (and layer norms) a plain one.  Returns the rows' log
        probabilities before the step (a view)."""
        if labels is None:
            raise ValueError("a training step needs labels")
        if self.pieces and entropy_weight:
            raise ValueError("a loss in pieces has no entropy")
        n, K, last = self._rows(x, labels), self.dims[-1], len(self.w) - 1
        inputs = self._forward(x, n, True)

        def below(l):                # where the gradient of layer l's input goes: the layer before's, or with norm the features'
            return self.dz[l - 1] if l else self.dx

        if self.pieces:
            i = self.dims[-2]
            B.vgg_fc_xent(self.dtype, n, i, K, inputs[last], self.operand[last], self.b[last], labels, self.logp, self.stats, self.ws)
            self.g_logp[:n].fill_(1.0 / n)
            B.vgg_fc_xent_bwd(self.dtype, B.F32, n, i, K, inputs[last], self.operand[last], self.b[last], labels, self.stats, self.g_logp,
                              below(last), self.dw[last], self.db[last], self.ws, relu_mask=last > 0 and not self.norm)
            self.logp[:n].neg_()
        else:
            B.vgg_log_probs(B.F32, n, K, self.logits, labels, 0, self.logp, self.entropy, None, None, self.stats, self.ws)
            self.g_logp[:n].fill_(-1.0 / n)
            self.g_entropy[:n].fill_(-entropy_weight / n)
            B.vgg_log_probs_bwd(B.F32, n, K, self.logits, labels, self.stats, self.entropy, self.g_logp,
                                self.g_entropy if entropy_weight else None, self.dz[-1])
        for l in reversed(range(len(self.w))):
            o, i = self.w[l].shape
            if not (l == last and self.pieces):
                B.vgg_fc_bwd(self.dtype, n, i, o, inputs[l], self.operand[l], self.dz[l], self.dw[l], self.db[l], below(l),
                             l > 0 and not self.norm, self.ws)
            p = self.dropout if l else 0.0
            if self.norm:
                B.vgg_layer_norm_bwd(self.dtype, B.F32, n, i, self.act[l - 1] if l else x, self.gamma[l], self.norm_stats[l], p, self.rng, l,
                                     below(l), below(l), self.dgamma[l], self.dbeta[l], l > 0, self.ws)
            elif p:
                B.vgg_dropout(B.F32, n, i, below(l), p, self.rng, l, below(l))
        for l, w in enumerate(self.w):
            B.vgg_muon_update(self.update_dtype, 1, *w.shape, self.ns_steps, w, self.dw[l], self.momentum[l], self.lr, self.mu, True,
                              self.weight_decay, self.ws)
        for t, g in zip(self.b + self.gamma + self.beta, self.db + self.dgamma + self.dbeta):
            B.vgg_sgd_update(t.numel(), t, g, self.bias_lr)
        if self.dropout:
            self.rng[1:].add_(1)
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
                z = self._scores() if l == last else self.act[l]
                B.vgg_fc_w4(self.dtype, n, i, o, self.group, self._input(l, a, n, False), c, s, self.b[l], z, B.F32 if l == last else self.dtype, l < last,
                            self.ws)
                a = z
        B.vgg_log_probs(B.F32, n, self.dims[-1], self.logits, labels, self.top, self.logp if labels is not None else None,
                        self.entropy, self.top_logp if self.top else None, self.top_idx if self.top else None, None, self.ws)
        return Answer(self.logp[:n] if labels is not None else None, self.entropy[:n], self.top_logp[:n] if self.top else None,
                      self.top_idx[:n] if self.top else None)
