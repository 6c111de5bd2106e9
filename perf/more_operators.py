"""What a head of tags is trained with, asked and served by, beside its layers and losses, as a program calls it.

Four kinds of pass:

  logp    log probabilities of the tags given with each image, entropy of the distribution over the vocabulary, and the
          likeliest tags: the answers alone, or with the gradients of x and w for given gradients of the log
          probabilities and entropies (training on a reward, or on several tags an image with an entropy term)
  muon    one step of gradient descent whose update is the momentum, orthogonalised by Newton-Schulz products, for a
          stack of matrices
  q8      y = x W^T from 8-bit weights with a scale for each output, x rounded to 8 bits with a scale for each row
  q8_glu  h = act(x Wg^T) * (x Wu^T) in the same way

`listed` spans one image to a large batch, `draw` spreads over the same ranges: 1 to 8192 rows, 64 to 8192 features,
1000 to 200000 words, up to 16 given tags and 32 likeliest ones, stacks of up to 2^28 values in all, in fp32 and bf16.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
ABC = (3.4445, -4.7750, 2.0315)     # of the Newton-Schulz step
MOMENTUM, STEPS, DECAY = 0.95, 5, 0.001


def _logp(N, D, V, T, K, dtype, train, masked, **name):
    return {"op": "logp", "N": N, "D": D, "V": V, "T": T, "K": K, "dtype": dtype, "train": train, "masked": masked, **name}


def _muon(count, rows, cols, dtype, nesterov, **name):
    return {"op": "muon", "count": count, "rows": rows, "cols": cols, "dtype": dtype, "nesterov": nesterov, **name}


def _q8(op, N, D, F, dtype, **name):
    return {"op": op, "N": N, "D": D, "F": F, "dtype": dtype, **name}


def listed():
    return [
        # one image asked for its ten likeliest tags: the vocabulary's weights stream by once
        _logp(1, 4096, 128000, 0, 10, "bf16", False, 0.0, name="logp_ask_bf16"),
        # a handful of images with up to three tags each, sizes that no tile divides, fp32
        _logp(7, 1021, 20011, 3, 5, "f32", False, 0.2, name="logp_few_f32"),
        # training a mini-batch of 192 images on several tags each
        _logp(192, 1024, 20011, 8, 0, "bf16", True, 0.3, name="logp_train_192_bf16"),
        # training a large batch over a large vocabulary, one tag an image, with the likeliest tags beside it
        _logp(8192, 4096, 128000, 1, 10, "bf16", True, 0.1, name="logp_train_bf16"),
        # the two small matrices of a hidden layer: launches and latency
        _muon(2, 256, 400, "f32", True, name="muon_small_f32"),
        # an untied layer, a matrix of filters for each of its 29 x 29 fields
        _muon(841, 2048, 128, "f32", True, name="muon_fields_f32"),
        # both matrices of a large hidden layer
        _muon(2, 8192, 4096, "bf16", True, name="muon_hidden_bf16"),
        # the weights of an odd vocabulary, without the look ahead
        _muon(1, 20011, 1021, "bf16", False, name="muon_words_bf16"),
        # one image through a gated layer of 8-bit weights: both matrices stream by once
        _q8("q8_glu", 1, 4096, 8192, "bf16", name="q8_glu_one_bf16"),
        # a large batch through it
        _q8("q8_glu", 8192, 4096, 8192, "bf16", name="q8_glu_large_bf16"),
        # scores of a mini-batch of 192 over a large odd vocabulary
        _q8("q8", 192, 4096, 100003, "bf16", name="q8_scores_192_bf16"),
        # a few rows of odd widths, fp32
        _q8("q8", 21, 1000, 2603, "f32", name="q8_few_f32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: often a multiple of 64, otherwise any number."""
    n = _log_int(rng, lo, hi)
    return max(lo, n // 64 * 64) if rng.random() < 0.5 else n


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if c["dtype"] == "bf16" else 1.6e14))


def draw(rng):
    most = _cost(listed()[3])
    while True:
        op = rng.choice(["logp", "logp", "muon", "muon", "q8", "q8_glu"])
        dtype = rng.choice(["f32", "bf16", "bf16"])
        if op == "logp":
            T, K = rng.choice([0, 1, 1, rng.randint(2, 16)]), rng.choice([0, 1, rng.randint(2, 32)])
            c = _logp(_log_int(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 1000, 200000), T, K, dtype,
                      T > 0 and rng.random() < 0.5, rng.choice([0.0, 0.1, 0.5]))
        elif op == "muon":
            rows, cols = _size(rng, 16, 8192), _size(rng, 16, 8192)
            c = _muon(_log_int(rng, 1, max(1, min(2000, (1 << 28) // (rows * cols)))), rows, cols, dtype,
                      rng.random() < 0.7)
        else:
            c = _q8(op, _log_int(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 50000), dtype)
        if _cost(c) <= most:
            return c


# ------------------------------------------------------------------------------------------------------------ inputs
def _to_8_bits(w):
    """Rows of 8-bit whole numbers, padded with zeros to whole blocks of 128, and the value of one for each row."""
    scale = w.abs().amax(dim=1)
    scale = (scale / torch.full_like(scale, 127.0)).clamp(min=2.0 ** -126)
    q = torch.zeros((w.shape[0], -(-w.shape[1] // 128) * 128), dtype=torch.int8, device=w.device)
    q[:, :w.shape[1]] = torch.round(w / scale[:, None]).clamp(-127, 127).to(torch.int8)
    return q, scale


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[c["dtype"]]

    def normal(shape, dtype, std):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    s = {"case": c}
    if c["op"] == "muon":
        shape = n, rows, cols = c["count"], c["rows"], c["cols"]
        r = min(8, rows, cols)

        def gradient(dtype):
            """A few strong directions and noise."""
            strong = torch.bmm(normal((n, rows, r), torch.float32, 1.0), normal((n, r, cols), torch.float32, 1.0))
            return strong.mul_(1e-3).add_(normal(shape, torch.float32, 1e-3)).to(dtype)

        s["w"], s["g"], s["m"] = normal(shape, dt, 1.0 / math.sqrt(cols)), gradient(dt), gradient(torch.float32).mul_(8.0)
        s["w_out"], s["m_out"] = torch.empty_like(s["w"]), torch.empty_like(s["m"])
        s["rate"] = 0.02 * math.sqrt(max(rows, cols))
        return s
    N, D = c["N"], c["D"]
    if c["op"] == "logp":
        V, T, K = c["V"], c["T"], c["K"]
        # from images that say little to images that leave hardly a choice
        s["x"] = normal((N, D), torch.float32, 1.0).mul_(
            torch.rand((N, 1), generator=gen, device="cuda").mul_(1.5).add_(0.25)).to(dt)
        s["w"] = normal((V, D), dt, 2.0 / math.sqrt(D))
        s["tags"] = None
        if T:
            # tags are used very unevenly, and images have different numbers of them; some have none
            t = torch.exp(torch.rand((N, T), generator=gen, device="cuda", dtype=torch.float64) * math.log(V))
            t = t.floor_().long().sub_(1).clamp_(0, V - 1)
            has = torch.randint(1, T + 1, (N, 1), generator=gen, device="cuda")
            has = torch.where(torch.rand((N, 1), generator=gen, device="cuda") < c["masked"], 0, has)
            s["tags"] = torch.where(torch.arange(T, device="cuda")[None, :] < has, t, -1)
        s["logp"] = torch.empty((N, T), device="cuda") if T else None
        s["entropy"] = torch.empty(N, device="cuda")
        s["top"] = torch.empty((N, K), dtype=torch.int64, device="cuda") if K else None
        s["top_logp"] = torch.empty((N, K), device="cuda") if K else None
        if c["train"]:
            s["dlogp"], s["dentropy"] = normal((N, T), torch.float32, 1.0 / N), normal((N,), torch.float32, 0.01 / N)
            s["state"] = torch.empty((N, 3), device="cuda")
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        return s
    F = c["F"]
    s["x"] = normal((N, D), dt, 1.0)
    for k in ("a", "b")[:2 if c["op"] == "q8_glu" else 1]:
        s["q" + k], s["s" + k] = _to_8_bits(normal((F, D), torch.float32, 1.0 / math.sqrt(D)))
    s["y"] = torch.empty((N, F), dtype=dt, device="cuda")
    return s


# --------------------------------------------------------------------------------------------------------- plain form
def _plain_logp(c, s):
    x, w, tags, K, N = s["x"].float(), s["w"].float(), s["tags"], c["K"], c["N"]
    l = x @ w.t()
    counts = (tags >= 0).any(dim=1) if c["T"] else torch.ones(N, dtype=torch.bool, device=x.device)
    top = l.amax(dim=1, keepdim=True)
    e = torch.exp(l - top)
    total = e.sum(dim=1, keepdim=True)
    log_total = torch.log(total)
    entropy = (log_total - (e * (l - top)).sum(dim=1, keepdim=True) / total)
    out = {"entropy": torch.where(counts, entropy[:, 0], 0.0)}
    if c["T"]:
        given = tags.clamp(min=0)
        logp = (l.gather(1, given) - top) - log_total
        out["logp"] = torch.where(tags >= 0, logp, 0.0)
    if K:
        # which of two near ones comes first is seen in 64 bits, equal ones in the vocabulary's order
        near = torch.topk(l, min(c["V"], K + 16), dim=1).indices.sort(dim=1).values
        fine = torch.bmm(s["w"][near].double(), s["x"].double()[:, :, None])[:, :, 0]
        order = torch.sort(fine, dim=1, descending=True, stable=True)
        at = order.indices[:, :K]
        out["top"] = torch.where(counts[:, None], near.gather(1, at), -1)
        top_logp = (fine.gather(1, at) - top) - log_total
        out["top_logp"] = torch.where(counts[:, None], top_logp, 0.0).float()
    if c["train"]:
        a = torch.where(tags >= 0, s["dlogp"], 0.0)
        b = torch.where(counts, s["dentropy"], 0.0)[:, None]
        p = e / total
        d = -p * (a.sum(dim=1, keepdim=True) + b * (((l - top) - log_total) + entropy))
        d = torch.where(counts[:, None], d, 0.0).scatter_add_(1, given, a)
        out["dx"], out["dw"] = (d @ w).to(s["x"].dtype), (d.t() @ x).to(s["x"].dtype)
    return out


def _plain_muon(c, s):
    g, m = s["g"].float(), MOMENTUM * s["m"] + s["g"].float()
    u = g + MOMENTUM * m if c["nesterov"] else m
    x = u / u.double().square().sum(dim=(1, 2), keepdim=True).sqrt().float()
    if c["rows"] > c["cols"]:
        x = x.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        a = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = ABC[0] * x + torch.bmm(ABC[1] * a + ABC[2] * torch.bmm(a, a), x)
    if c["rows"] > c["cols"]:
        x = x.transpose(1, 2)
    return {"w": ((1.0 - DECAY) * s["w"].float() - s["rate"] * x).to(s["w"].dtype), "m": m}


def _plain_q8(c, s):
    x = s["x"].float()
    scale = x.abs().amax(dim=1, keepdim=True)
    # by a tensor: by a number, a multiplication with its rounded reciprocal would take the division's place
    scale = (scale / torch.full_like(scale, 127.0)).clamp(min=2.0 ** -126)
    # halves are told from their neighbours in 64 bits
    q = torch.round(x.double() / scale.double()).clamp(-127, 127).float()
    y = [(q @ s["q" + k][:, :c["D"]].float().t()) * scale * s["s" + k] for k in ("a", "b") if "q" + k in s]
    return {"y": (y[0] if len(y) == 1 else y[0] / (1.0 + torch.exp(-y[0])) * y[1]).to(s["x"].dtype)}


# --------------------------------------------------------------------------------------------------------------- pass
def _scratch(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _own_logp(lc, c, s, dtype):
    N, D, V, T, K = (c[k] for k in ("N", "D", "V", "T", "K"))
    ws = _scratch(lc.logp_workspace_bytes(N, D, V, T, K, dtype, c["train"]))
    lc.logp_fwd(s["x"], s["w"], s["tags"], s["logp"], s["entropy"], s["top"], s["top_logp"], s.get("state"), dtype, ws)
    if c["train"]:
        lc.logp_bwd(s["x"], s["w"], s["tags"], s["logp"], s["state"], s["dlogp"], s["dentropy"], s["dx"], s["dw"], dtype, ws)
    return {k: s[k] for k in ("logp", "entropy", "top", "top_logp", "dx", "dw") if s.get(k) is not None}


def _own_muon(lc, c, s, dtype):
    ws = _scratch(lc.muon_workspace_bytes(c["count"], c["rows"], c["cols"], dtype))
    lc.muon_step(s["w"], s["g"], s["m"], s["w_out"], s["m_out"], s["rate"], DECAY, MOMENTUM, c["nesterov"], STEPS, dtype, ws)
    return {"w": s["w_out"], "m": s["m_out"]}


def _own_q8(lc, c, s, dtype):
    ws = _scratch(lc.q8_workspace_bytes(c["N"], c["D"], c["F"], dtype))
    if c["op"] == "q8":
        lc.q8_matmul(s["x"], s["qa"], s["sa"], s["y"], dtype, ws)
    else:
        lc.q8_glu_fwd(s["x"], s["qa"], s["sa"], s["qb"], s["sb"], s["y"], lc.LC_ACT_SILU, dtype, ws)
    return {"y": s["y"]}


def run(s):
    c = s["case"]
    if own:
        import paper_1502_03409_amd as lc

        dtype = lc.LC_BF16 if c["dtype"] == "bf16" else lc.LC_F32
        return {"logp": _own_logp, "muon": _own_muon}.get(c["op"], _own_q8)(lc, c, s, dtype)
    return {"logp": _plain_logp, "muon": _plain_muon}.get(c["op"], _plain_q8)(c, s)


# -------------------------------------------------------------------------------------------------------------- floor
def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "muon":
        n, small, large = c["count"], min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
        # reads w, g and the momentum, writes the weights and the momentum; of the symmetric products one half
        return {"bytes": n * small * large * (3 * es + 8),
                "flops": n * STEPS * (small * (small + 1) * large + small * (small + 1) * small + 2 * small * small * large)}
    N, D = c["N"], c["D"]
    if c["op"] == "logp":
        V, T, K = c["V"], c["T"], c["K"]
        rows = 12 * N * T + 4 * N + 12 * N * K
        if not c["train"]:
            return {"bytes": es * (N * D + V * D) + rows, "flops": 2 * N * D * V}
        # the backward pass needs the gradients given for each row on the way in, dx and dw on the way out
        return {"bytes": 2 * es * (N * D + V * D) + rows + 4 * N * T + 4 * N, "flops": 6 * N * D * V}
    F, two = c["F"], 2 if c["op"] == "q8_glu" else 1
    return {"bytes": es * (N * D + N * F) + two * (F * D + 4 * F), "flops": 2 * two * N * D * F}


# ------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The same outputs from the definitions, with derivatives by differentiation of the double precision values."""
    c, s = case, prepare(case, seed)
    if c["op"] == "muon":
        m = s["m"].double() * MOMENTUM + s["g"].double()
        u = torch.add(s["g"].double(), m, alpha=MOMENTUM) if c["nesterov"] else m
        x = u / torch.linalg.vector_norm(u, dim=(1, 2), keepdim=True)
        tall = c["rows"] > c["cols"]
        eye = torch.eye(min(c["rows"], c["cols"]), dtype=torch.float64, device=x.device)
        for _ in range(STEPS):
            gram = x.mT.contiguous() @ x if tall else x @ x.mT.contiguous()
            p = ABC[0] * eye + gram @ (ABC[1] * eye + ABC[2] * gram)
            x = x @ p if tall else p @ x
        return {"w": s["w"].double() * (1.0 - DECAY) - x * s["rate"], "m": m}
    if c["op"] == "logp":
        x, w = (s[k].double().requires_grad_(c["train"]) for k in ("x", "w"))
        lp = torch.log_softmax(torch.nn.functional.linear(x, w), dim=1)
        some = (s["tags"] >= 0).any(dim=1) if c["T"] else torch.ones(c["N"], dtype=torch.bool, device=x.device)
        entropy = torch.special.entr(lp.exp()).sum(dim=1).where(some, torch.zeros((), dtype=torch.float64, device=x.device))
        out = {"entropy": entropy.detach()}
        if c["T"]:
            logp = torch.take_along_dim(lp, s["tags"].clamp(min=0), dim=1).masked_fill(s["tags"] < 0, 0.0)
            out["logp"] = logp.detach()
        if c["K"]:
            best = torch.topk(lp.detach(), c["K"], dim=1)
            out["top"] = best.indices.masked_fill(~some[:, None], -1)
            out["top_logp"] = best.values.masked_fill(~some[:, None], 0.0)
        if c["train"]:
            cost = (logp * s["dlogp"].double()).sum() + (entropy * s["dentropy"].double()).sum()
            out["dx"], out["dw"] = torch.autograd.grad(cost, (x, w))
        return out
    x = s["x"].double()
    amax = x.abs().amax(dim=1)
    scale = torch.clamp((amax / torch.full_like(amax, 127.0)).float().double(), min=2.0 ** -126)
    q = torch.clamp(torch.round(x / scale[:, None]), -127, 127) * scale[:, None]
    y = [torch.nn.functional.linear(q, s["q" + k][:, :c["D"]].double() * s["s" + k].double()[:, None])
         for k in ("a", "b") if "q" + k in s]
    return {"y": y[0] if len(y) == 1 else torch.nn.functional.silu(y[0]) * y[1]}
