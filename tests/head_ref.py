"""The head's operators in 64 bits, from their definitions (torch on whatever device the inputs are), and the tolerances of the
kernels' tests."""
import math

import torch

ACTS = ("sigmoid", "silu", "gelu")


def act(name, g):
    """act(g), act'(g)."""
    if name == "gelu":
        phi = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if name == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def glu(x, wg, wu, name):
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    return act(name, g)[0] * u, g, u


def glu_grads(x, wg, wu, dh, name):
    x, wg, wu, dh = (t.double() for t in (x, wg, wu, dh))
    g, u = x @ wg.t(), x @ wu.t()
    a, da = act(name, g)
    dg, du = dh * u * da, dh * a
    return dg @ wg + du @ wu, dg.t() @ x, du.t() @ x


def xent(x, w, target, scale=None):
    """loss, cost, dx, dw; masked rows of x are never looked at."""
    counts = target >= 0
    x, w = torch.where(counts[:, None], x.double(), 0.0), w.double()
    s = torch.where(counts, scale.double() if scale is not None else 1.0 / max(1, int(counts.sum())), 0.0)
    l = x @ w.t()
    lse = torch.logsumexp(l, dim=1)
    t = target.clamp(min=0)
    loss = torch.where(counts, lse - l.gather(1, t[:, None])[:, 0], 0.0)
    d = torch.exp(l - lse[:, None])
    # p_t - 1 without cancellation
    d.scatter_(1, t[:, None], torch.expm1(l.gather(1, t[:, None]) - lse[:, None]))
    d = torch.where(counts[:, None], d * s[:, None], 0.0)
    return loss, (loss * s).sum(), d @ w, d.t() @ x


def tol(dtype, K, roundings):
    """Bound on the relative error (2-norms) of a product over K terms.  fp32: one rounding of 2^-24 for each of the six partial
    products of a term, adding up like a random walk, and a margin of 16 for what is computed before and after.  bf16: each
    rounding to bf16 on the way, the result's own included, costs at most 2^-8 (eight significant bits)."""
    if dtype == torch.float32:
        return 2.0 ** -24 * (math.sqrt(6 * K) + 16)
    return roundings * 2.0 ** -8 + 2.0 ** -24 * math.sqrt(K)


def check(what, got, want, bound):
    """2-norm of the difference within `bound` of the result's, and no single value off by more than 64 bounds of the larger of
    itself and the root mean square (a lost or doubled tile is off by all of it)."""
    got, want = got.double().cpu(), want.double().cpu()
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and torch.equal(torch.isinf(got), inf), what
    fine = torch.isfinite(want)
    got, want = got[fine], want[fine]
    if not want.numel():
        return
    d, size = got - want, float(want.norm())
    assert float(d.norm()) <= bound * size, (what, float(d.norm()) / max(size, 1e-300), bound)
    rms = size / math.sqrt(want.numel())
    if rms:
        worst = float((d.abs() / want.abs().clamp(min=rms)).max())
        assert worst <= 64 * bound, (what, worst, bound)
