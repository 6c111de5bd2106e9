"""The operators of a supervised head on learned features, as a program that trains or serves one calls them.

Features x [N, D] go through a gated hidden layer and a softmax cross entropy over a vocabulary of tags; the gradients
of all tensors are clipped by their global norm.  Three kinds of pass:

  glu   h = act(x Wg^T) * (x Wu^T): the forward pass alone (answering), or with the backward pass (training)
  xent  loss_n = log sum_v exp(x_n . w_v) - x_n . w_t(n) and its weighted sum over the rows whose target is not
        negative: the loss alone (evaluation), or with the gradients of x and w (training)
  clip  the 2-norm over all values of a list of tensors, and every tensor times min(1, max_norm / norm)

`listed` spans one image to a large batch, `draw` spreads over the same ranges: 1 to 8192 rows, 64 to 8192 features,
hidden layers of 64 to 16384, vocabularies of 1000 to 200000, 1 to 60 tensors of up to 2^28 values, in fp32 and bf16.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _glu(N, D, F, act, dtype, train, **name):
    return {"op": "glu", "N": N, "D": D, "F": F, "act": act, "dtype": dtype, "train": train, **name}


def _xent(N, D, V, dtype, train, masked, weighted, **name):
    return {"op": "xent", "N": N, "D": D, "V": V, "dtype": dtype, "train": train, "masked": masked,
            "weighted": weighted, **name}


def _clip(tensors, total, dtype, clips, shape_seed, **name):
    return {"op": "clip", "tensors": tensors, "total": total, "dtype": dtype, "clips": clips, "shape_seed": shape_seed,
            **name}


def listed():
    return [
        # one image asked for: both weights stream by once
        _glu(1, 4096, 8192, "silu", "bf16", False, name="glu_one_bf16"),
        # a handful of images, sizes that no tile divides, fp32
        _glu(7, 1000, 2603, "gelu", "f32", False, name="glu_few_f32"),
        # one mini-batch of 192 images on the way to answers
        _glu(192, 4096, 8192, "silu", "bf16", False, name="glu_batch_bf16"),
        # training the hidden layer on a large batch
        _glu(8192, 4096, 8192, "silu", "bf16", True, name="glu_train_bf16"),
        # training in fp32 with odd sizes throughout
        _glu(1537, 1021, 2055, "gelu", "f32", True, name="glu_train_odd_f32"),
        # a few rows scored against a large odd vocabulary
        _xent(5, 4096, 100003, "bf16", False, 0.0, False, name="xent_score_bf16"),
        # training on a mini-batch of 192 with some rows unlabelled: the vocabulary's weights dominate
        _xent(192, 1024, 20011, "bf16", True, 0.2, False, name="xent_train_192_bf16"),
        # training on a large batch over a large vocabulary
        _xent(8192, 4096, 128000, "bf16", True, 0.1, False, name="xent_train_bf16"),
        # training in fp32 with weights for the rows
        _xent(1000, 768, 30011, "f32", True, 0.3, True, name="xent_train_f32"),
        # gradients of a small head: launches and latency
        _clip(3, 100_000, "f32", True, 1, name="clip_small_f32"),
        # gradients of a deep model: many tensors of both types and very different sizes
        _clip(60, 50_000_000, "mixed", True, 2, name="clip_many"),
        # gradients of a large untied layer, far beyond the caches
        _clip(4, 1_000_000_000, "mixed", True, 3, name="clip_large"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: often a multiple of 64, otherwise any number."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if c["dtype"] == "bf16" else 1.6e14))


def draw(rng):
    most = 0.02
    while True:
        op = rng.choice(["glu", "glu", "xent", "xent", "clip"])
        dtype = rng.choice(["f32", "bf16", "bf16"])
        train = rng.random() < 0.6
        if op == "glu":
            c = _glu(_log_int(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 16384),
                     rng.choice(["sigmoid", "silu", "gelu"]), dtype, train)
        elif op == "xent":
            c = _xent(_log_int(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 1000, 200000), dtype, train,
                      rng.choice([0.0, 0.1, 0.5]), rng.random() < 0.3)
        else:
            tensors = _log_int(rng, 1, 60)
            c = _clip(tensors, max(4 * tensors, _log_int(rng, 1000, 1 << 28)), rng.choice(["f32", "bf16", "mixed"]),
                      rng.random() < 0.7, rng.randrange(1 << 20))
        if _cost(c) <= most and 3072 not in c.values():
            return c


# ------------------------------------------------------------------------------------------------------------ inputs
def _shapes(c):
    """Sizes and types of a list of gradients: sizes over three orders of magnitude, the sum as the case says."""
    gen = torch.Generator().manual_seed(c["shape_seed"])
    part = torch.exp(torch.rand(c["tensors"], generator=gen, dtype=torch.float64) * 7.0)
    sizes = [max(1, int(v)) for v in (part / part.sum() * c["total"]).tolist()]
    kinds = ["f32", "bf16"] if c["dtype"] == "mixed" else [c["dtype"]]
    return [(n, DTYPE[kinds[i % len(kinds)]]) for i, n in enumerate(sizes)]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, dtype, std):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    s = {"case": c}
    if c["op"] == "clip":
        shapes = _shapes(c)
        s["grads"] = [normal((n,), dt, 0.02 * (1 + i % 3)) for i, (n, dt) in enumerate(shapes)]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]
        s["norm"] = torch.empty(1, device="cuda")
        size = math.sqrt(sum(n * (0.02 * (1 + i % 3)) ** 2 for i, (n, _) in enumerate(shapes)))
        s["max_norm"] = size * (0.3 if c["clips"] else 2.0)
        return s
    dt = DTYPE[c["dtype"]]
    N, D = c["N"], c["D"]
    if c["op"] == "glu":
        F = c["F"]
        s["x"] = normal((N, D), dt, 1.0)
        s["wg"], s["wu"] = normal((F, D), dt, 1.0 / math.sqrt(D)), normal((F, D), dt, 1.0 / math.sqrt(D))
        s["h"] = torch.empty((N, F), dtype=dt, device="cuda")
        if c["train"]:
            s["dh"] = normal((N, F), dt, 1.0 / N)
            s["gu"] = torch.empty((N, 2, F), dtype=dt, device="cuda")
            s["dx"], s["dwg"], s["dwu"] = (torch.empty_like(s[k]) for k in ("x", "wg", "wu"))
        return s
    V = c["V"]
    s["x"], s["w"] = normal((N, D), dt, 1.0), normal((V, D), dt, 2.0 / math.sqrt(D))
    # tags are used very unevenly: few of them make up most of the targets
    u = torch.rand(N, generator=gen, device="cuda", dtype=torch.float64)
    t = torch.exp(u * math.log(V)).floor_().long().sub_(1).clamp_(0, V - 1)
    drop = torch.rand(N, generator=gen, device="cuda") < c["masked"]
    s["target"] = torch.where(drop, torch.full_like(t, -1), t)
    s["scale"] = torch.rand(N, generator=gen, device="cuda").add_(0.5).div_(N) if c["weighted"] else None
    s["loss"], s["cost"] = torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    if c["train"]:
        s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    return s


# --------------------------------------------------------------------------------------------------------- plain form
def _act(name, g):
    """act(g) and its derivative."""
    if name == "gelu":
        half = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * half, half + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-g))
    if name == "sigmoid":
        return sig, sig * (1.0 - sig)
    return g * sig, sig * (1.0 + g * (1.0 - sig))


def _plain_glu(c, s):
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _act(c["act"], g)
    h = (a * u).to(s["x"].dtype)
    if not c["train"]:
        return {"h": h}
    dh = s["dh"].float()
    dg, du = dh * u * da, dh * a
    dt = s["x"].dtype
    return {"h": h, "dx": (dg @ wg + du @ wu).to(dt), "dwg": (dg.t() @ x).to(dt), "dwu": (du.t() @ x).to(dt)}


def _plain_xent(c, s):
    x, w, t = s["x"].float(), s["w"].float(), s["target"]
    counts = t >= 0
    at = t.clamp(min=0)[:, None]
    logits = x @ w.t()
    top = logits.amax(dim=1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(dim=1, keepdim=True)
    loss = torch.where(counts, (torch.log(total) + top - logits.gather(1, at))[:, 0], 0.0)
    scale = s["scale"] if s["scale"] is not None else 1.0 / counts.sum().clamp(min=1).float()
    scale = torch.where(counts, scale, 0.0)
    out = {"loss": loss, "cost": (scale * loss).sum().reshape(1)}
    if not c["train"]:
        return out
    d = (e / total).scatter_add_(1, at, torch.full_like(total, -1.0)) * scale[:, None]
    dt = s["x"].dtype
    return {**out, "dx": (d @ w).to(dt), "dw": (d.t() @ x).to(dt)}


def _plain_clip(s):
    flat = torch.cat([g.float() for g in s["grads"]])
    norm = flat.square().sum().sqrt()
    coef = torch.clamp(s["max_norm"] / norm, max=1.0)
    return {"norm": norm.reshape(1), "out": [(g.float() * coef).to(g.dtype) for g in s["grads"]]}


# --------------------------------------------------------------------------------------------------------------- pass
def _scratch(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _own_glu(lc, c, s):
    dtype = lc.LC_BF16 if c["dtype"] == "bf16" else lc.LC_F32
    act = {"sigmoid": lc.LC_ACT_SIGMOID, "silu": lc.LC_ACT_SILU, "gelu": lc.LC_ACT_GELU}[c["act"]]
    N, D, F = c["N"], c["D"], c["F"]
    ws = _scratch(lc.glu_workspace_bytes(N, D, F, dtype, c["train"]))
    lc.glu_fwd(s["x"], s["wg"], s["wu"], s["h"], s.get("gu"), act, dtype, ws)
    if not c["train"]:
        return {"h": s["h"]}
    lc.glu_bwd(s["x"], s["wg"], s["wu"], s["gu"], s["dh"], s["dx"], s["dwg"], s["dwu"], act, dtype, ws)
    return {k: s[k] for k in ("h", "dx", "dwg", "dwu")}


def _own_xent(lc, c, s):
    dtype = lc.LC_BF16 if c["dtype"] == "bf16" else lc.LC_F32
    ws = _scratch(lc.xent_workspace_bytes(c["N"], c["D"], c["V"], dtype, c["train"]))
    if not c["train"]:
        lc.xent_fwd(s["x"], s["w"], s["target"], s["scale"], s["loss"], s["cost"], dtype, ws)
        return {"loss": s["loss"], "cost": s["cost"]}
    lc.xent_fwd_bwd(s["x"], s["w"], s["target"], s["scale"], s["loss"], s["cost"], s["dx"], s["dw"], dtype, ws)
    return {k: s[k] for k in ("loss", "cost", "dx", "dw")}


def _own_clip(lc, s):
    ws = _scratch(lc.grad_clip_workspace_bytes(s["grads"]))
    lc.grad_clip(s["grads"], s["out"], s["max_norm"], s["norm"], ws)
    return {"norm": s["norm"], "out": s["out"]}


def run(s):
    c = s["case"]
    if own:
        import paper_1502_03409_amd as lc

        return _own_glu(lc, c, s) if c["op"] == "glu" else _own_xent(lc, c, s) if c["op"] == "xent" else _own_clip(lc, s)
    return _plain_glu(c, s) if c["op"] == "glu" else _plain_xent(c, s) if c["op"] == "xent" else _plain_clip(s)


# -------------------------------------------------------------------------------------------------------------- floor
def work(case):
    c = case
    if c["op"] == "clip":
        moved = sum(n * (4 if dt == torch.float32 else 2) for n, dt in _shapes(c))
        return {"bytes": 2 * moved, "flops": 3 * c["total"]}
    es, N, D = (4 if c["dtype"] == "f32" else 2), c["N"], c["D"]
    if c["op"] == "glu":
        F = c["F"]
        fwd = N * D + 2 * F * D + N * F
        # the backward pass reads dh and writes dx and both weight gradients
        return {"bytes": es * (fwd + (N * F + N * D + 2 * F * D if c["train"] else 0)),
                "flops": 4 * N * D * F * (3 if c["train"] else 1)}
    V = c["V"]
    return {"bytes": es * (N * D + V * D) * (2 if c["train"] else 1) + 12 * N + (4 * N if c["weighted"] else 0),
            "flops": 2 * N * D * V * (3 if c["train"] else 1)}


# ------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The same outputs from the definitions, with derivatives by differentiation of the double precision loss."""
    c, s = case, prepare(case, seed)
    if c["op"] == "clip":
        norm = math.sqrt(sum(float(torch.dot(g.double(), g.double())) for g in s["grads"]))
        k = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
        return {"norm": torch.tensor([norm], dtype=torch.float64), "out": [g.double() * k for g in s["grads"]]}
    x = s["x"].double().requires_grad_(c["train"])
    if c["op"] == "glu":
        wg, wu = (s[k].double().requires_grad_(c["train"]) for k in ("wg", "wu"))
        fn = {"sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[c["act"]]
        h = fn(torch.nn.functional.linear(x, wg)) * torch.nn.functional.linear(x, wu)
        if not c["train"]:
            return {"h": h}
        dx, dwg, dwu = torch.autograd.grad(h, (x, wg, wu), s["dh"].double())
        return {"h": h.detach(), "dx": dx, "dwg": dwg, "dwu": dwu}
    w = s["w"].double().requires_grad_(c["train"])
    loss = torch.nn.functional.cross_entropy(torch.nn.functional.linear(x, w), s["target"], ignore_index=-1,
                                             reduction="none")
    if s["scale"] is None:
        cost = loss.sum() / max(1, int((s["target"] >= 0).sum()))
    else:
        cost = torch.dot(loss, s["scale"].double())
    out = {"loss": loss.detach(), "cost": cost.detach().reshape(1)}
    if not c["train"]:
        return out
    dx, dw = torch.autograd.grad(cost, (x, w))
    return {**out, "dx": dx, "dw": dw}
