"""What a classifier's dense layers are trained with, served from and answer, as timed and compared cases.

Three kinds of work, each through the functions of binding (`own`) or in elementary torch operations (not `own`):

  scores    class scores to log probabilities: of given classes, with the entropy and the most likely alternatives of
            every row ("answer"), or with the gradient of the scores ("train")
  w4        dense layers from 4-bit weights with group scales: the product ("product"), or the weights' rounding to
            codes and scales and the values that these stand for ("quantize")
  muon      orthogonalised updates by Newton-Schulz products: of matrices of one shape ("orthogonalize"), or the whole
            optimiser step with momentum on fp32 parameters ("update")

A masked class has the score -inf.  A row without a class left has the log probabilities -inf, the entropy 0 and the
gradient 0; alternatives that a row lacks are -inf at class -1.  Ties go to the lowest class.  Labels outside the
classes have the log probability 0 and no gradient.

4-bit codes hold a sign and 0, 0.5, 1, 1.5, 2, 3, 4 or 6; a group of consecutive inputs of one output shares a bf16
scale, a sixth of its largest magnitude.  Rows of codes are padded to 32 codes, two to a byte, the even one low.
"""
import math

import torch

own = False

HIDDEN, CLASSES = 4096, 1000
STEPS, LR, MU, DECAY = 5, 0.02, 0.95, 0.01
NS = (3.4445, -4.7750, 2.0315)   # coefficients of x, x^3 and x^5 in one Newton-Schulz step
EPS = 1e-7                       # added to the Frobenius norm that a matrix is divided by
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one image's answer: class probabilities of its 1000 scores and the five best, the smallest call of serving
        {"name": "scores_f32_1x1000", "kind": "scores", "op": "answer", "dtype": "f32", "N": 1, "K": CLASSES, "top": 5, "masked": False},
        # the same for the paper's largest batch
        {"name": "scores_f32_100x1000", "kind": "scores", "op": "answer", "dtype": "f32", "N": 100, "K": CLASSES, "top": 5, "masked": False},
        # few rows over a large, odd set of classes, a tenth of them masked
        {"name": "scores_bf16_4x200003", "kind": "scores", "op": "answer", "dtype": "bf16", "N": 4, "K": 200003, "top": 20, "masked": True},
        # training over many classes: log probabilities, entropy and the gradient of the scores
        {"name": "scores_train_bf16_4096x32768", "kind": "scores", "op": "train", "dtype": "bf16", "N": 4096, "K": 32768, "top": 0, "masked": False},
        # the widest dense layer for one image: 51 MB of codes stream past one row
        {"name": "w4_bf16_1x25088x4096", "kind": "w4", "op": "product", "dtype": "bf16", "N": 1, "In": 25088, "Out": HIDDEN, "group": 128, "relu": True},
        # the last layer in fp32 at the paper's middle batch, the finest groups
        {"name": "w4_f32_10x4096x1000", "kind": "w4", "op": "product", "dtype": "f32", "N": 10, "In": HIDDEN, "Out": CLASSES, "group": 32, "relu": False},
        # the middle layer at the paper's largest batch
        {"name": "w4_bf16_100x4096x4096", "kind": "w4", "op": "product", "dtype": "bf16", "N": 100, "In": HIDDEN, "Out": HIDDEN, "group": 64, "relu": True},
        # rounding the widest layer's weights, once per trained model
        {"name": "w4_quantize_25088x4096", "kind": "w4", "op": "quantize", "dtype": "f32", "N": 1, "In": 25088, "Out": HIDDEN, "group": 128, "relu": False},
        # the second convolution's filters as a matrix: a chain of the smallest products
        {"name": "ortho_bf16_64x576", "kind": "muon", "op": "orthogonalize", "dtype": "bf16", "batch": 1, "rows": 64, "cols": 576},
        # the seven widest convolutions of one shape together
        {"name": "ortho_bf16_7x512x4608", "kind": "muon", "op": "orthogonalize", "dtype": "bf16", "batch": 7, "rows": 512, "cols": 4608},
        # the optimiser's step for the last dense layer: rows that fill no tile
        {"name": "muon_f32_1000x4096", "kind": "muon", "op": "update", "dtype": "f32", "batch": 1, "rows": CLASSES, "cols": HIDDEN},
        # ... and for the first, which holds most of the network's parameters
        {"name": "muon_f32_4096x25088", "kind": "muon", "op": "update", "dtype": "f32", "batch": 1, "rows": HIDDEN, "cols": 25088},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["scores", "w4", "muon"])
    dtype = rng.choice(["bf16", "f32"])
    if kind == "scores":
        op = rng.choice(["answer", "train"])
        n = _log(rng, 1, 4096)
        k = _log(rng, 2, min(262144, (1 << 27) // (n if dtype == "bf16" else 2 * n)))
        return {"kind": kind, "op": op, "dtype": dtype, "N": n, "K": k, "top": min(k, _log(rng, 1, 64)) if op == "answer" else 0,
                "masked": rng.random() < 0.4}
    if kind == "w4":
        op = rng.choice(["product", "product", "product", "quantize"])
        return {"kind": kind, "op": op, "dtype": dtype if op == "product" else "f32", "N": _log(rng, 1, 128) if op == "product" else 1,
                "In": _log(rng, 32, 25088), "Out": _log(rng, 10, 4096), "group": rng.choice([32, 64, 128]), "relu": rng.random() < 0.5}
    op = rng.choice(["orthogonalize", "update"])
    while True:
        c = {"kind": kind, "op": op, "dtype": dtype if op == "orthogonalize" else "f32", "batch": _log(rng, 1, 8), "rows": _log(rng, 16, 8192),
             "cols": _log(rng, 16, 25088)}
        if work(c)["flops"] <= 1e12:
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


def _scores_inputs(case, seed):
    """Scores of a classifier that is sure of some rows; one label in twenty is none; upstream gradients of a mean loss."""
    d, n, k = _Draw(seed), case["N"], case["K"]
    z = d.normal(n, k, std=2.5)
    labels = d.integers(0, k, n)
    z += 8.0 * (torch.arange(k, device="cuda") == labels[:, None]) * (d.uniform(n, 1) < 0.5)
    if case["masked"]:
        z.masked_fill_(d.uniform(1, k) < 0.1, -math.inf)
    labels = torch.where(d.uniform(n) < 0.05, torch.full_like(labels, -1), labels) if n > 1 else labels
    return {"z": z.to(_td(case)), "labels": labels, "g_logp": -(0.5 + d.uniform(n)) / n, "g_entropy": d.normal(n, std=0.05 / n)}


def _w4_inputs(case, seed):
    """He-normal weights; activations after a ReLU."""
    d, n, i, o = _Draw(seed), case["N"], case["In"], case["Out"]
    return {"w": d.normal(o, i, std=math.sqrt(2.0 / i)), "a": d.normal(n, i).clamp_min_(0).to(_td(case)), "b": d.normal(o, std=0.01)}


def _muon_inputs(case, seed):
    """Gradients of dense layers: the products of a batch's activations (after a ReLU) and output gradients, and noise; the
    momentum of earlier ones, wider spread; He-normal parameters."""
    d, b, m, n = _Draw(seed), case["batch"], case["rows"], case["cols"]

    def gradient(examples, noise):
        out = torch.empty((b, m, n), device="cuda")
        for k in range(b):
            out[k] = d.normal(m, examples, std=1.0 / examples) @ d.normal(examples, n).clamp_min_(0)
        return out.add_(d.normal(b, m, n, std=noise))

    s = {"grad": gradient(100, 0.02)}
    if case["op"] == "update":
        s["momentum"] = gradient(400, 0.2)
        s["theta"] = d.normal(b, m, n, std=math.sqrt(2.0 / n))
    else:
        s["grad"] = s["grad"].to(_td(case))
    return s


def _codes_of(w, group):
    """Codes [Out][In], as numbers 0..15, and bf16 scales [Out][groups] of fp32 weights: the nearest values, ties to the
    even code.  The bounds between codes are exact products of the scale."""
    o, i = w.shape
    groups = -(-i // group)
    v = torch.zeros((o, groups * group), device=w.device).index_copy_(1, torch.arange(i, device=w.device), w).view(o, groups, group)
    scales = (v.abs().amax(2) * torch.tensor(1 / 6, dtype=torch.float32)).to(torch.bfloat16)
    s, mag = scales.float()[:, :, None], v.abs()
    at = (mag > 0.25 * s).byte()
    at += mag.ge(0.75 * s) & (s > 0)
    at += mag > 1.25 * s
    at += mag.ge(1.75 * s) & (s > 0)
    at += mag > 2.5 * s
    at += mag.ge(3.5 * s) & (s > 0)
    at += mag > 5.0 * s
    at += 8 * (v < 0).byte()
    return at.view(o, -1)[:, :i].contiguous(), scales


def _packed(codes):
    o, i = codes.shape
    full = torch.zeros((o, -(-i // 32) * 32), dtype=torch.uint8, device=codes.device)
    full[:, :i] = codes
    return (full[:, 0::2] | (full[:, 1::2] << 4)).contiguous()


def _values(codes, scales, group):
    """The fp32 values of codes [Out][In] and their scales."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    return grid[codes.long()] * scales.float().repeat_interleave(group, 1)[:, :codes.shape[1]]


def _bytes(n):
    return torch.empty((max(int(n), 16),), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    kind = case["kind"]
    if kind == "scores":
        n, k = case["N"], case["K"]
        s = dict(_scores_inputs(case, seed), case=case)
        for name, shape in (("logp", (n,)), ("entropy", (n,)), ("top_logp", (n, case["top"])), ("stats", (n, 2))):
            s[name] = torch.empty(shape, device="cuda")
        s["top_idx"] = torch.empty((n, case["top"]), dtype=torch.int32, device="cuda")
        if case["op"] == "train":
            s["dz"] = torch.empty((n, k), dtype=_td(case), device="cuda")
        return s
    if kind == "w4":
        i, o, g = case["In"], case["Out"], case["group"]
        t = _w4_inputs(case, seed)
        s = {"case": case}
        if case["op"] == "product":
            codes, s["scales"] = _codes_of(t["w"], g)
            s["codes"], s["a"], s["b"] = _packed(codes), t["a"], t["b"]
            s["z"] = torch.empty((case["N"], o), dtype=_td(case), device="cuda")
        else:
            s["w"] = t["w"]
            s["codes"] = torch.empty((o, -(-i // 32) * 16), dtype=torch.uint8, device="cuda")
            s["scales"] = torch.empty((o, -(-i // g)), dtype=torch.bfloat16, device="cuda")
            s["values"] = torch.empty((o, i), device="cuda")
        return s
    s = dict(_muon_inputs(case, seed), case=case)
    if case["op"] == "orthogonalize":
        s["out"] = torch.empty_like(s["grad"])
    return s


# ------------------------------------------------------------------------------------------- the calls
def _binding(s, query):
    """The binding, the library's name of the case's type and, kept from the first pass on, the workspace it asks for."""
    from paper_1810_09868_amd import binding as B
    dt = B.BF16 if s["case"]["dtype"] == "bf16" else B.F32
    if "ws" not in s:
        s["ws"] = _bytes(query(B, dt))
    return B, dt, s["ws"]


def _own_scores(s):
    c = s["case"]
    n, k, top = c["N"], c["K"], c["top"]
    B, dt, ws = _binding(s, lambda B, dt: B.vgg_log_probs_workspace_bytes(dt, n, k, top))
    B.vgg_log_probs(dt, n, k, s["z"], s["labels"], top, s["logp"], s["entropy"], s["top_logp"] if top else None,
                    s["top_idx"] if top else None, s["stats"], ws)
    if c["op"] == "answer":
        return {"logp": s["logp"], "entropy": s["entropy"], "top_logp": s["top_logp"], "top_idx": s["top_idx"]}
    B.vgg_log_probs_bwd(dt, n, k, s["z"], s["labels"], s["stats"], s["entropy"], s["g_logp"], s["g_entropy"], s["dz"])
    return {"logp": s["logp"], "entropy": s["entropy"], "dz": s["dz"]}


def _own_w4(s):
    c = s["case"]
    n, i, o, g = c["N"], c["In"], c["Out"], c["group"]
    if c["op"] == "product":
        B, dt, ws = _binding(s, lambda B, dt: B.vgg_fc_w4_workspace_bytes(dt, n, i, o, g))
        B.vgg_fc_w4(dt, n, i, o, g, s["a"], s["codes"], s["scales"], s["b"], s["z"], dt, c["relu"], ws)
        return s["z"]
    B, _, _ = _binding(s, lambda B, dt: 16)
    B.vgg_fc_w4_quantize(i, o, g, s["w"], s["codes"], s["scales"])
    B.vgg_fc_w4_dequantize(i, o, g, s["codes"], s["scales"], s["values"])
    return {"values": s["values"], "scales": s["scales"]}


def _own_muon(s):
    c = s["case"]
    b, m, n = c["batch"], c["rows"], c["cols"]
    if c["op"] == "orthogonalize":
        B, dt, ws = _binding(s, lambda B, dt: B.vgg_orthogonalize_workspace_bytes(dt, b, m, n))
        B.vgg_orthogonalize(dt, b, m, n, STEPS, s["grad"], s["out"], ws)
        return s["out"]
    B, dt, ws = _binding(s, lambda B, dt: B.vgg_muon_workspace_bytes(dt, b, m, n))
    B.vgg_muon_update(dt, b, m, n, STEPS, s["theta"], s["grad"], s["momentum"], LR, MU, True, DECAY, ws)
    return {"theta": s["theta"], "momentum": s["momentum"]}


def _plain_scores(s):
    c, z, labels = s["case"], s["z"].float(), s["labels"].long()
    k, top = c["K"], c["top"]
    here = (labels >= 0) & (labels < k)
    most = z.amax(1, keepdim=True)
    left = most > -math.inf                              # rows with a class
    shifted = torch.where(left, z - most, -math.inf)     # (-inf - -inf is NaN)
    e = shifted.exp()
    total = e.sum(1, keepdim=True)
    lp = shifted - total.log()
    lp = torch.where(left, lp, -math.inf)
    p = e / total.clamp_min(1.0)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    logp = torch.where(here, lp.gather(1, labels.clamp(0, k - 1)[:, None])[:, 0], 0.0)
    if c["op"] == "answer":
        # values, then classes, in one sortable whole number: the order of floats as integers, lower classes first
        bits = (z + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 32) + (k - 1 - torch.arange(k, device=z.device))
        idx = k - 1 - (key.topk(top, dim=1).values & 0xFFFFFFFF)
        best = lp.gather(1, idx)
        return {"logp": logp, "entropy": entropy, "top_logp": best, "top_idx": torch.where(best > -math.inf, idx, -1).int()}
    g = torch.where(here, s["g_logp"], 0.0)[:, None]
    dz = -g * p - s["g_entropy"][:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), 0.0)
    mark = torch.arange(k, device=z.device) == labels[:, None]
    dz = torch.where(mark & (z > -math.inf), dz + g, dz)
    return {"logp": logp, "entropy": entropy, "dz": dz.to(s["z"].dtype)}


def _plain_w4(s):
    c = s["case"]
    i, g = c["In"], c["group"]
    if c["op"] == "quantize":
        codes, scales = _codes_of(s["w"], g)
        return {"values": _values(codes, scales, g), "scales": scales}
    codes = torch.stack((s["codes"] & 15, s["codes"] >> 4), 2).flatten(1)[:, :i]
    z = s["a"].float() @ _values(codes, s["scales"], g).t() + s["b"]
    return (z.clamp_min(0) if c["relu"] else z).to(s["a"].dtype)


def _orthogonal(u):
    """Newton-Schulz steps on [batch][rows][cols]; the shorter side's Gram matrix."""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    a, b, c = NS
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2).contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2).contiguous() if tall else x


def _plain_muon(s):
    if s["case"]["op"] == "orthogonalize":
        return _orthogonal(s["grad"].float()).to(s["grad"].dtype)
    g, m, theta = s["grad"], s["momentum"], s["theta"]
    m.mul_(MU).add_(g)
    update = _orthogonal(g + MU * m)
    theta.mul_(1 - LR * DECAY).sub_(LR * math.sqrt(max(1.0, theta.shape[1] / theta.shape[2])) * update)
    return {"theta": theta, "momentum": m}


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own_scores(s) if kind == "scores" else _own_w4(s) if kind == "w4" else _own_muon(s)
    return _plain_scores(s) if kind == "scores" else _plain_w4(s) if kind == "w4" else _plain_muon(s)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    kind, es = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "scores":
        n, k = case["N"], case["K"]
        # the gradient needs the scores once more (or kept on the chip, which is not counted on: written once)
        return {"bytes": n * k * es * (2 if case["op"] == "train" else 1) + n * (16 + 8 * case["top"]), "flops": 4 * n * k * (2 if case["op"] == "train" else 1)}
    if kind == "w4":
        n, i, o, groups = case["N"], case["In"], case["Out"], -(-case["In"] // case["group"])
        coded = o * (-(-i // 32) * 16 + 2 * groups)
        if case["op"] == "quantize":
            return {"bytes": 8 * o * i + 2 * coded, "flops": 9 * o * i}
        return {"bytes": coded + (n * i + n * o) * es + 4 * o, "flops": 2 * n * i * o}
    b, m, n = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # a step: the Gram matrix and its square (symmetric: half of them) and the product with the matrix
    flops = b * STEPS * (m * m * n + m * m * m + 2 * m * m * n)
    return {"bytes": b * m * n * (2 * es if case["op"] == "orthogonalize" else 20), "flops": flops}


# --------------------------------------------------------------------------------------- 64-bit values
def _exact_scores(case, seed):
    t = _scores_inputs(case, seed)
    z, k = t["z"].double(), case["K"]
    there = torch.isfinite(z)
    any_there = there.any(1, keepdim=True)
    lse = torch.logsumexp(z.masked_fill(~any_there, 0.0), 1, keepdim=True)
    lp = (z - lse).masked_fill(~there, -math.inf)
    p = lp.exp()
    plp = (p * lp.masked_fill(~there, 0.0))
    entropy = -plp.sum(1)
    ok = (t["labels"] >= 0) & (t["labels"] < k)
    at = t["labels"].long().clamp(0, k - 1)[:, None]
    logp = lp.gather(1, at).squeeze(1).masked_fill(~ok, 0.0)
    if case["op"] == "answer":
        order = lp.sort(dim=1, descending=True, stable=True)
        best = order.values[:, :case["top"]]
        idx = order.indices[:, :case["top"]].masked_fill(best == -math.inf, -1)
        return {"logp": logp, "entropy": entropy, "top_logp": best, "top_idx": idx.int()}
    g = t["g_logp"].double().masked_fill(~ok, 0.0)[:, None]
    hot = torch.zeros_like(p).scatter_(1, at, 1.0).masked_fill(~there, 0.0)
    dz = g * (hot - p * any_there) - t["g_entropy"].double()[:, None] * (plp + p * entropy[:, None])
    return {"logp": logp, "entropy": entropy, "dz": dz}


def _exact_w4(case, seed):
    t, g = _w4_inputs(case, seed), case["group"]
    i, values, scales = case["In"], [], []
    marks = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device="cuda")
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    for j in range(0, i, g):
        w = t["w"][:, j:j + g]
        s = (w.abs().amax(1, keepdim=True) * torch.tensor(1 / 6, dtype=torch.float32)).to(torch.bfloat16)
        r = w.double().abs() / s.double().clamp_min(1e-300)
        lower = torch.bucketize(r, marks)               # a tie keeps the lower value ...
        upper = torch.bucketize(r, marks, right=True)   # ... or takes the upper one: the one of even code
        code = torch.where(lower % 2 == 0, lower, upper)
        values.append(grid[code] * s.double() * w.double().sign())
        scales.append(s)
    w = torch.cat(values, 1)
    if case["op"] == "quantize":
        return {"values": w, "scales": torch.cat(scales, 1).double()}
    z = t["a"].double() @ w.t() + t["b"].double()
    return torch.relu(z) if case["relu"] else z


def _exact_muon(case, seed):
    t = {k: v.double() for k, v in _muon_inputs(case, seed).items()}
    u = t["grad"]
    if case["op"] == "update":
        t["momentum"] = MU * t["momentum"] + t["grad"]
        u = t["grad"] + MU * t["momentum"]
    done = []
    for x in u:
        flip = x.shape[0] > x.shape[1]
        x = x.t() if flip else x
        x = x / (torch.linalg.vector_norm(x) + EPS)
        for _ in range(STEPS):
            g = x @ x.t()
            x = NS[0] * x + NS[1] * (g @ x) + NS[2] * (g @ (g @ x))
        done.append(x.t() if flip else x)
    o = torch.stack(done)
    if case["op"] == "orthogonalize":
        return o
    rate = LR * max(1.0, case["rows"] / case["cols"]) ** 0.5
    return {"theta": (1 - LR * DECAY) * t["theta"] - rate * o, "momentum": t["momentum"]}


def exact(case, seed):
    with torch.no_grad():
        return {"scores": _exact_scores, "w4": _exact_w4, "muon": _exact_muon}[case["kind"]](case, seed)
