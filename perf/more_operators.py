"""What the training of a classifier's dense layers needs around its products, as timed and compared cases.

Three kinds of work, each through the functions of binding (`own`) or in elementary torch operations (not `own`):

  norm   layer norm of rows, with dropout of what leaves it ("forward"), and with the gradients of the rows, the scale and
         the shift ("train"); in training the rows may be what a ReLU left, whose derivative their gradient then takes too
  drop   dropout of a layer's activations ("forward") and of their gradient as well ("train")
  xent   a dense layer over many classes and its softmax cross entropy, row by row ("loss"), and with the gradients of
         activations, weights and biases for a weight of every row's loss ("train")

Dropout's random numbers are those of Philox 4x32-10 (Salmon, Moraes, Dror and Shaw: Parallel random numbers: as easy as
1, 2, 3; SC 2011) with the seed as its key and the counter (column / 8, row, low word of the step, layer << 16 | bits 32 to 47
of the step): eight numbers of 16 bits, low halves first, for eight neighbouring columns.  A value is dropped where its
number is less than 65536 p, rounded; others are divided by the share that is kept.  Seed and step are numbers in device
memory.

A class whose bias is -inf is masked.  Labels outside the classes have the loss 0 and no gradient; a masked label's loss
is inf, and masked classes have no gradient.
"""
import math

import torch

own = False

HIDDEN, CLASSES, FEATURES = 4096, 1000, 25088
EPS = 1e-5


def listed():
    return [
        # one image's features between two dense layers: the smallest call
        {"name": "norm_f32_1x4096", "kind": "norm", "op": "forward", "dtype": "f32", "N": 1, "C": HIDDEN, "pad": 0, "p": 0.0, "relu": False},
        # training at the paper's largest batch: what a hidden layer's ReLU left, half of it dropped
        {"name": "norm_train_bf16_100x4096", "kind": "norm", "op": "train", "dtype": "bf16", "N": 100, "C": HIDDEN, "pad": 0, "p": 0.5, "relu": True},
        # many short, odd rows that are parts of longer ones
        {"name": "norm_train_f32_50001x333", "kind": "norm", "op": "train", "dtype": "f32", "N": 50001, "C": 333, "pad": 3, "p": 0.1, "relu": False},
        # the flattened features of a large batch
        {"name": "norm_train_bf16_8192x25088", "kind": "norm", "op": "train", "dtype": "bf16", "N": 8192, "C": FEATURES, "pad": 0, "p": 0.0, "relu": True},
        # dropout of a hidden layer at the paper's largest batch, forward and backward
        {"name": "drop_train_bf16_100x4096", "kind": "drop", "op": "train", "dtype": "bf16", "N": 100, "C": HIDDEN, "pad": 0, "p": 0.5},
        # ... of rows that no vector divides
        {"name": "drop_f32_3001x4099", "kind": "drop", "op": "forward", "dtype": "f32", "N": 3001, "C": 4099, "pad": 0, "p": 0.1},
        # ... of a large batch's features
        {"name": "drop_train_bf16_8192x25088", "kind": "drop", "op": "train", "dtype": "bf16", "N": 8192, "C": FEATURES, "pad": 0, "p": 0.5},
        # one image's loss over the network's classes: the smallest call
        {"name": "xent_bf16_1x4096x1000", "kind": "xent", "op": "loss", "dtype": "bf16", "N": 1, "In": HIDDEN, "K": CLASSES, "masked": False},
        # the network's last layer and its loss at the paper's largest batch
        {"name": "xent_train_f32_100x4096x1000", "kind": "xent", "op": "train", "dtype": "f32", "N": 100, "In": HIDDEN, "K": CLASSES, "masked": False},
        # few rows over a large, odd set of classes, a tenth of them masked: the weights stream past the rows
        {"name": "xent_train_bf16_4x4096x200003", "kind": "xent", "op": "train", "dtype": "bf16", "N": 4, "In": HIDDEN, "K": 200003, "masked": True},
        # fp32 at sizes that fill no tile
        {"name": "xent_train_f32_1000x1001x50001", "kind": "xent", "op": "train", "dtype": "f32", "N": 1000, "In": 1001, "K": 50001, "masked": False},
        # many rows over many classes: products of full tiles, scores that would fill gigabytes
        {"name": "xent_train_bf16_8192x2048x131072", "kind": "xent", "op": "train", "dtype": "bf16", "N": 8192, "In": 2048, "K": 131072, "masked": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "drop", "xent", "xent"])
    dtype, op = rng.choice(["bf16", "f32"]), rng.choice(["forward", "train"])
    if kind != "xent":
        n = _log(rng, 1, 65536)
        # (rows of a few values have next to no gradient left once their mean and width are taken out)
        c = _log(rng, 8 if kind == "norm" else 1, min(FEATURES, (1 << 26) // n))
        if rng.random() < 0.5 and c > 16:
            c -= c % 8
        case = {"kind": kind, "op": op, "dtype": dtype, "N": n, "C": c, "pad": rng.choice([0, 0, 8, 3]), "p": rng.choice([0.0, 0.1, 0.25, 0.5])}
        if kind == "norm":
            case["relu"] = op == "train" and rng.random() < 0.5
        elif case["p"] == 0.0:
            case["p"] = 0.5
        return case
    while True:
        c = {"kind": kind, "op": "loss" if op == "forward" else op, "dtype": dtype, "N": _log(rng, 1, 8192), "In": _log(rng, 16, HIDDEN),
             "K": _log(rng, 2, 262144), "masked": rng.random() < 0.3}
        if rng.random() < 0.5 and c["In"] > 64:
            c["In"] -= c["In"] % 64
        if c["N"] * c["In"] * c["K"] <= (1 << 39 if dtype == "f32" else 1 << 41) and c["K"] * c["In"] <= 1 << 29:
            return c


# ---------------------------------------------------------------------------------------------- inputs
class _Draw:
    """Seeded draws on the GPU, in call order."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32) * std

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def integers(self, lo, hi, n):
        return torch.randint(lo, hi, (n,), generator=self.g, device="cuda", dtype=torch.int32)


def _td(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rng_state(d):
    """Seed and step: any 64 bits, and a step past 32."""
    return torch.randint(-(1 << 62), 1 << 62, (2,), generator=d.g, device="cuda") & torch.tensor([-1, (1 << 34) - 1], device="cuda")


def _rows_inputs(case, seed):
    """Activations with an offset and a width of their own in every row, after a ReLU where the case has one, and the
    gradient of what is made of them; rows of C out of C + pad numbers."""
    d, n, c, ld = _Draw(seed), case["N"], case["C"], case["C"] + case["pad"]
    s = {"rng": _rng_state(d), "layer": 1 + int(seed) % 5}
    x = d.normal(n, ld) * (0.5 + d.uniform(n, 1)) + d.normal(n, 1)
    s["x"] = (x.clamp_min_(0) if case.get("relu") else x).to(_td(case))[:, :c]
    if case["op"] == "train":
        s["dy"] = d.normal(n, ld, std=1.0 / n).to(_td(case))[:, :c]
    if case["kind"] == "norm":
        s["gamma"], s["beta"] = 1 + d.normal(c, std=0.2), d.normal(c, std=0.1)
    return s


def _xent_inputs(case, seed):
    """Normalised activations, half of them near their label's weights; one label in twenty is none; weights of a mean loss."""
    d, n, i, k = _Draw(seed), case["N"], case["In"], case["K"]
    w, a, labels = d.normal(k, i, std=2.5 / math.sqrt(i)), d.normal(n, i), d.integers(0, k, n)
    near = w[labels.long()]
    a += 8.0 * (d.uniform(n, 1) < 0.5) * near / near.square().sum(1, keepdim=True)
    bias = d.normal(k, std=0.1)
    if case["masked"]:
        bias.masked_fill_(d.uniform(k) < 0.1, -math.inf)
    labels = torch.where(d.uniform(n) < 0.05, torch.full_like(labels, -1), labels) if n > 1 else labels
    return {"a": a.to(_td(case)), "w": w.to(_td(case)), "bias": bias, "labels": labels, "g_loss": (0.5 + d.uniform(n)) / n}


def prepare(case, seed):
    f32 = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
    typed = lambda *shape: torch.empty(shape, dtype=_td(case), device="cuda")  # noqa: E731
    train, n = case["op"] == "train", case["N"]
    if case["kind"] == "xent":
        i, k = case["In"], case["K"]
        s = dict(_xent_inputs(case, seed), case=case, loss=f32(n), stats=f32(n, 2))
        if train:
            s.update(da=typed(n, i), dw=typed(k, i), db=f32(k))
        return s
    c = case["C"]
    s = dict(_rows_inputs(case, seed), case=case, y=typed(n, c))
    if train:
        s["dx"] = typed(n, c)
    if case["kind"] == "norm":
        s["stats"] = f32(n, 2)
        if train:
            s.update(dgamma=f32(c), dbeta=f32(c))
    return s


# ------------------------------------------------------------------------------------------- the calls
def _binding(s, query):
    """The binding, the library's name of the case's type and, kept from the first pass on, the workspace it asks for."""
    from paper_1810_09868_amd import binding as B
    dt = B.BF16 if s["case"]["dtype"] == "bf16" else B.F32
    if "ws" not in s:
        s["ws"] = torch.empty((max(int(query(B, dt)), 16),), dtype=torch.uint8, device="cuda")
    return B, dt, s["ws"]


def _own_norm(s):
    c = s["case"]
    n, cols, ld, p = c["N"], c["C"], c["C"] + c["pad"], c["p"]
    B, dt, ws = _binding(s, lambda B, dt: B.vgg_layer_norm_bwd_workspace_bytes(dt, dt, n, cols))
    B.vgg_layer_norm(dt, n, cols, s["x"], s["gamma"], s["beta"], EPS, p, s["rng"] if p else None, s["layer"], s["y"], s["stats"], ldx=ld)
    if c["op"] == "forward":
        return {"y": s["y"], "stats": s["stats"]}
    B.vgg_layer_norm_bwd(dt, dt, n, cols, s["x"], s["gamma"], s["stats"], p, s["rng"] if p else None, s["layer"], s["dy"], s["dx"],
                         s["dgamma"], s["dbeta"], c["relu"], ws, ldx=ld, lddy=ld)
    return {"y": s["y"], "stats": s["stats"], "dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _own_drop(s):
    c = s["case"]
    n, cols, ld = c["N"], c["C"], c["C"] + c["pad"]
    B, dt, _ = _binding(s, lambda B, dt: 16)
    B.vgg_dropout(dt, n, cols, s["x"], c["p"], s["rng"], s["layer"], s["y"], ldx=ld)
    if c["op"] == "forward":
        return s["y"]
    B.vgg_dropout(dt, n, cols, s["dy"], c["p"], s["rng"], s["layer"], s["dx"], ldx=ld)
    return {"y": s["y"], "dx": s["dx"]}


def _own_xent(s):
    c = s["case"]
    n, i, k, train = c["N"], c["In"], c["K"], c["op"] == "train"
    B, dt, ws = _binding(s, lambda B, dt: max(B.vgg_fc_xent_workspace_bytes(dt, n, i, k), B.vgg_fc_xent_bwd_workspace_bytes(dt, n, i, k) if train else 0))
    B.vgg_fc_xent(dt, n, i, k, s["a"], s["w"], s["bias"], s["labels"], s["loss"], s["stats"], ws)
    if not train:
        return s["loss"]
    B.vgg_fc_xent_bwd(dt, dt, n, i, k, s["a"], s["w"], s["bias"], s["labels"], s["stats"], s["g_loss"], s["da"], s["dw"], s["db"], ws)
    return {"loss": s["loss"], "da": s["da"], "dw": s["dw"], "db": s["db"]}


def _kept(rng, layer, n, c, p):
    """[n][c] truth values: which elements dropout keeps."""
    low, dev = 0xFFFFFFFF, rng.device
    blocks = -(-c // 8)
    x0 = torch.arange(blocks, device=dev).expand(n, blocks)
    x1 = torch.arange(n, device=dev)[:, None].expand(n, blocks)
    x2 = (rng[1] & low).expand(n, blocks)
    x3 = ((rng[1] >> 32 & 0xFFFF) | layer << 16).expand(n, blocks)
    k0, k1 = rng[0] & low, rng[0] >> 32 & low
    for _ in range(10):
        a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57   # (products wrap at 64 bits: their bits are those of unsigned ones)
        x0, x1, x2, x3 = (b >> 32 & low) ^ x1 ^ k0, b & low, (a >> 32 & low) ^ x3 ^ k1, a & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    numbers = torch.stack((x0 & 0xFFFF, x0 >> 16, x1 & 0xFFFF, x1 >> 16, x2 & 0xFFFF, x2 >> 16, x3 & 0xFFFF, x3 >> 16), 2)
    return (numbers >= _dropped_of_65536(p)).view(n, blocks * 8)[:, :c]


def _dropped_of_65536(p):
    return int(math.floor(p * 65536 + 0.5))


def _scale(p):
    return 65536.0 / (65536 - _dropped_of_65536(p))


def _plain_norm(s):
    c, x, p = s["case"], s["x"].float(), s["case"]["p"]
    n, cols = x.shape
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / (centred.square().mean(1, keepdim=True) + EPS).sqrt()
    xh = centred * rstd
    y = xh * s["gamma"] + s["beta"]
    keep = _kept(s["rng"], s["layer"], n, cols, p) if p else None
    if p:
        y = torch.where(keep, y * _scale(p), 0.0)
    out = {"y": y.to(s["x"].dtype), "stats": torch.cat((mean, rstd), 1)}
    if c["op"] == "forward":
        return out
    g = s["dy"].float()
    if p:
        g = torch.where(keep, g * _scale(p), 0.0)
    out["dgamma"], out["dbeta"] = (g * xh).sum(0), g.sum(0)
    g = g * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    out["dx"] = (torch.where(x > 0, dx, 0.0) if c["relu"] else dx).to(s["x"].dtype)
    return out


def _plain_drop(s):
    c = s["case"]
    keep = _kept(s["rng"], s["layer"], c["N"], c["C"], c["p"])
    y = torch.where(keep, s["x"].float() * _scale(c["p"]), 0.0).to(s["x"].dtype)
    if c["op"] == "forward":
        return y
    return {"y": y, "dx": torch.where(keep, s["dy"].float() * _scale(c["p"]), 0.0).to(s["x"].dtype)}


def _plain_xent(s):
    c, labels, a, w = s["case"], s["labels"].long(), s["a"].float(), s["w"].float()
    here = (labels >= 0) & (labels < c["K"])
    at = labels.clamp(0, c["K"] - 1)[:, None]
    z = a @ w.t() + s["bias"]
    most = z.amax(1, keepdim=True)
    most = torch.where(most > -math.inf, most, 0.0)      # (a row without a class)
    z -= most
    zl = z.gather(1, at)
    e = z.exp().scatter_(1, at, 0.0)                     # the others' exponentials: what is left of a label that is all but certain
    rest, el = e.sum(1, keepdim=True), zl.exp()
    total = rest + el
    loss = torch.where(zl == 0, rest.log1p(), torch.where(zl > -math.inf, total.log() - zl, math.inf))[:, 0]
    loss = torch.where(here, loss, 0.0)
    if c["op"] == "loss":
        return loss
    share = torch.where(here, s["g_loss"], 0.0)[:, None] / total.clamp_min(1e-30)
    dz = e.mul_(share).scatter_(1, at, torch.where(zl > -math.inf, -rest * share, 0.0))
    return {"loss": loss, "da": (dz @ w).to(s["a"].dtype), "dw": (dz.t() @ a).to(s["w"].dtype), "db": dz.sum(0)}


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own_norm(s) if kind == "norm" else _own_drop(s) if kind == "drop" else _own_xent(s)
    return _plain_norm(s) if kind == "norm" else _plain_drop(s) if kind == "drop" else _plain_xent(s)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    es, train, n = 2 if case["dtype"] == "bf16" else 4, case["op"] == "train", case["N"]
    if case["kind"] == "xent":
        i, k = case["In"], case["K"]
        # the scores once for the loss; with gradients they would be kept at the least: three products
        return {"bytes": (n * i + k * i) * es * (2 if train else 1) + 4 * k * (2 if train else 1) + n * (16 if train else 8),
                "flops": 2 * n * i * k * (3 if train else 1)}
    c = case["C"]
    values = n * c * es * (4 if train else 2)
    if case["kind"] == "drop":
        return {"bytes": values + 16, "flops": n * c * (10 if train else 9)}
    return {"bytes": values + 8 * n + 8 * c * (2 if train else 1), "flops": n * c * (24 if train else 8)}


# --------------------------------------------------------------------------------------- 64-bit values
def _philox_numbers(seed, step, layer, rows, blocks):
    """Eight 16-bit numbers [rows][blocks][8] by long multiplication in halves of 16 bits."""
    def mul(x, m):
        lo, hi = x & 0xFFFF, x >> 16
        mlo, mhi = m & 0xFFFF, m >> 16
        t = lo * mlo
        mid = hi * mlo + (t >> 16)
        mid2 = lo * mhi + (mid & 0xFFFF)
        return hi * mhi + (mid >> 16) + (mid2 >> 16), (mid2 & 0xFFFF) << 16 | t & 0xFFFF

    counter = [torch.arange(blocks, device="cuda").repeat(rows, 1), torch.arange(rows, device="cuda").view(-1, 1).repeat(1, blocks),
               torch.full((rows, blocks), step % (1 << 32), device="cuda"),
               torch.full((rows, blocks), layer * 65536 + (step >> 32) % 65536, device="cuda")]
    key = [seed % (1 << 32), (seed >> 32) % (1 << 32)]
    for r in range(10):
        h0, l0 = mul(counter[0], 0xD2511F53)
        h1, l1 = mul(counter[2], 0xCD9E8D57)
        counter = [h1 ^ counter[1] ^ key[0], l1, h0 ^ counter[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    return torch.stack([(v >> 16 * half) & 0xFFFF for v in counter for half in (0, 1)], -1)


def _exact_factor(t, case):
    """What dropout multiplies by, [N][C]: 0 or one over the share that is kept."""
    p = case["p"]
    if p == 0:
        return 1.0
    seed, step = (int(v) for v in t["rng"].cpu())
    out, blocks = [], (case["C"] + 7) // 8
    numbers = _philox_numbers(seed, step, t["layer"], case["N"], blocks).flatten(1)[:, :case["C"]]
    dropped = round(p * 65536)
    return (numbers >= dropped).double() / (1 - dropped / 65536)


def _exact_norm(case, seed):
    t = _rows_inputs(case, seed)
    x, factor = t["x"].double(), _exact_factor(t, case)
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    rstd = (var + EPS).rsqrt()
    h = (x - mean) * rstd
    gamma = t["gamma"].double()
    out = {"y": torch.addcmul(t["beta"].double(), h, gamma) * factor, "stats": torch.cat([mean, rstd], 1)}
    if case["op"] == "train":
        g = t["dy"].double() * factor
        out["dbeta"] = g.sum(0)
        out["dgamma"] = (g * h).sum(0)
        g *= gamma
        along = (g * h).sum(1, keepdim=True) / case["C"]
        dx = (g - g.sum(1, keepdim=True) / case["C"] - h * along) * rstd
        out["dx"] = dx.masked_fill(x <= 0, 0.0) if case["relu"] else dx
    return out


def _exact_drop(case, seed):
    t = _rows_inputs(case, seed)
    factor = _exact_factor(t, case)
    y = t["x"].double() * factor
    return y if case["op"] == "forward" else {"y": y, "dx": t["dy"].double() * factor}


def _exact_xent(case, seed):
    t = {k: v.double() if v.is_floating_point() else v for k, v in _xent_inputs(case, seed).items()}
    n, k = case["N"], case["K"]
    z = torch.addmm(t["bias"], t["a"], t["w"].t())
    lse = torch.logsumexp(z, 1)
    rows = torch.arange(n, device="cuda")
    ok = (t["labels"] >= 0) & (t["labels"] < k)
    labels = torch.where(ok, t["labels"], 0).long()
    open_label = torch.isfinite(z[rows, labels])
    loss = torch.where(ok, torch.where(open_label, lse - z[rows, labels], math.inf), 0.0)
    if case["op"] == "loss":
        return loss
    g = torch.where(ok, t["g_loss"], 0.0)
    dz = torch.nan_to_num(torch.exp_(z.sub_(lse[:, None])), nan=0.0)    # (a row without a class)
    dz[rows, labels] -= open_label.double()
    dz *= g[:, None]
    return {"loss": loss, "da": dz @ t["w"], "dw": dz.t() @ t["a"], "db": dz.sum(0)}


def exact(case, seed):
    with torch.no_grad():
        return {"norm": _exact_norm, "drop": _exact_drop, "xent": _exact_xent}[case["kind"]](case, seed)
