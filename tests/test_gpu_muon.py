"""muon_step against its definition in 64 bits.

Tolerances follow the roundings through the steps, all in 2-norms over a matrix.  Held values are rounded by at most r of themselves: fp16
2^-11, two fp16 2^-22; a sum of K products in fp32 is off by about 2^-24 sqrt(3 K) of the operands' norms.  With S = X X^T + shift and
P = c S S + rest, in first order
    dS <= 2 r |X|_2 |X|_F + r |S|_F,   dP <= 2 c |S|_2 dS + r |P|_F,   dX' <= L dX + dP |X|_2 + r |X'|_F
(|.|_2 the largest singular value), where L = 3.4445 bounds the derivative of the step at any X whose singular values lie in [0, 1.203]."""
import math

import pytest
import torch

import paper_1502_03409_amd as lc

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
TYPES = [torch.float32, torch.bfloat16]
# sides around 8, 16, 64, 128 and 256, wide, tall and square, single rows and columns
SIZES = [(1, 1, 1), (1, 1, 7), (2, 9, 1), (1, 1, 300), (3, 8, 8), (5, 17, 30), (2, 64, 64), (3, 65, 40), (2, 128, 129), (1, 300, 100), (2, 100, 300),
         (1, 257, 260), (2, 520, 33), (1, 31, 1111), (1, 400, 640)]


def ids(t):
    return "bf16" if t == torch.bfloat16 else "f32"


def code(t):
    return lc.LC_BF16 if t == torch.bfloat16 else lc.LC_F32


def orthogonalised(u, steps, dtype, bounds=False):
    """The result for each matrix and a bound on the 2-norm of its error.  `bounds`: the largest singular values of X and S by their bounds, 1.203
    and 1.18, where finding them would take long."""
    r = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22
    small = min(u.shape[-2:])
    size = u.square().sum(dim=(1, 2), keepdim=True).sqrt()
    x = torch.where(size > 0, u / size, 0.0)
    if u.shape[1] > u.shape[2]:
        x = x.mT
    x = x.contiguous()
    eye = torch.eye(small, dtype=torch.float64, device=u.device)

    def fro(t):
        return t.square().sum(dim=(1, 2)).sqrt()

    def largest(t):
        return torch.linalg.matrix_norm(t, 2) if not bounds else 1.18 if t is s else 1.203

    err = (r + 2.0 ** -22) * fro(x)
    for _ in range(steps):
        s = x @ x.mT + B / (2 * C) * eye
        p = C * s @ s + (A - B * B / (4 * C)) * eye
        y = p @ x
        sums = 2.0 ** -24 * (math.sqrt(3 * max(u.shape[1:])) + 4)
        ds = (2 * r + sums) * largest(x) * fro(x) + r * fro(s)
        dp = 2 * C * largest(s) * ds + (r + sums) * fro(p) * 1.5
        err = A * err + (dp + sums * fro(p)) * largest(x) + r * fro(y)
        x = y
    return (x.mT if u.shape[1] > u.shape[2] else x), err


def definition(w, g, m, rate, decay, mu, nesterov, steps, bounds=False):
    rate, decay, mu = (float(torch.tensor(v, dtype=torch.float32)) for v in (rate, decay, mu))   # the entry point takes fp32 numbers
    m1 = mu * m.double() + g.double()
    u = g.double() + mu * m1 if nesterov else m1
    o, err = orthogonalised(u, steps, w.dtype, bounds)
    return m1, o, err, (1 - decay) * w.double() - rate * o


def draw(shape, dtype, seed, std=1.0, rank=None):
    gen = torch.Generator().manual_seed(seed)
    t = torch.randn(shape, generator=gen, dtype=torch.float64) * std
    if rank:
        t = t * 0.05 + torch.randn((*shape[:-1], rank), generator=gen, dtype=torch.float64) @ torch.randn((*shape[:-2], rank, shape[-1]), generator=gen, dtype=torch.float64) * std
    return t.to(dtype).cuda()


def scratch(shape, dtype):
    n = lc.muon_workspace_bytes(*shape, code(dtype))
    return torch.full((n // 4 + 64,), float("nan"), device="cuda")


def step(w, g, m, rate=0.3, decay=0.01, mu=0.9, nesterov=True, steps=5, in_place=False):
    w, m = w.clone(), m.clone()
    wo, mo = (None, None) if in_place else (torch.full_like(w, float("nan")), torch.full_like(m, float("nan")))
    lc.muon_step(w, g, m, wo, mo, rate, decay, mu, nesterov, steps, code(w.dtype), scratch(tuple(w.shape), w.dtype))
    return (w, m) if in_place else (wo, mo)


def check(got, w, g, m, rate=0.3, decay=0.01, mu=0.9, nesterov=True, steps=5, bounds=False):
    m1, o, err, w1 = definition(w, g, m, rate, decay, mu, nesterov, steps, bounds)
    assert ((got[1].double() - m1).abs() <= 2.0 ** -24 * m1.abs() + 2.0 ** -149).all()
    half = 2.0 ** -8 if w.dtype == torch.bfloat16 else 2.0 ** -24
    off = (got[0].double() - w1).square().sum(dim=(1, 2)).sqrt()
    # the result's rounding, and three in fp32 on the way to it
    size = w.double().square().sum(dim=(1, 2)).sqrt() + abs(rate) * o.square().sum(dim=(1, 2)).sqrt()
    bound = abs(rate) * err + (half + 2.0 ** -22) * size
    print("error over bound", float((off / bound.clamp(min=1e-300)).max()), "relative", float((err / o.square().sum(dim=(1, 2)).sqrt().clamp(min=1e-300)).max()))
    assert (off <= bound).all()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("steps", [1, 5])     # one: the bound is near what is lost, so that no plane or tile can be missing
@pytest.mark.parametrize("shape", SIZES, ids=str)
def test_values(shape, steps, dtype):
    print(f"case muon {shape} {dtype}", flush=True)
    w, g, m = draw(shape, dtype, 1, 0.5), draw(shape, dtype, 2), draw(shape, torch.float32, 3, 4.0)
    got = step(w, g, m, steps=steps)
    check(got, w, g, m, steps=steps)
    again = step(w, g, m, steps=steps, in_place=True)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("shape", [(2, 130, 70), (2, 70, 260)], ids=str)
@pytest.mark.parametrize("kw", [dict(nesterov=False), dict(steps=1), dict(steps=2), dict(steps=8), dict(mu=0.0), dict(decay=0.0, rate=-1.0), dict(decay=1.0)], ids=str)
def test_arguments(shape, kw, dtype):
    w, g, m = draw(shape, dtype, 4, 0.5), draw(shape, dtype, 5, rank=3), draw(shape, torch.float32, 6, 2.0, rank=3)
    check(step(w, g, m, **kw), w, g, m, **kw)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_singular_values_come_near_one(dtype):
    """From the definition alone: five steps take singular values above 0.02 of the norm into [0.6, 1.25]; columns and rows stay orthogonal."""
    g = draw((1, 96, 200), dtype, 7)
    w, m = torch.zeros_like(g), torch.zeros(g.shape, device="cuda")
    o = step(w, g, m, rate=-1.0, decay=0.0)[0][0].double()
    s = torch.linalg.svdvals(o)
    assert float(s.min()) > 0.6 and float(s.max()) < 1.25


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_magnitudes_do_not_matter(dtype):
    """Powers of two cancel, down to where the values themselves lose bits and up to where their squares leave fp32."""
    shape = (1, 40, 72)
    w, g, m = draw(shape, dtype, 8), draw(shape, dtype, 9), torch.zeros(shape, device="cuda")
    first = step(w, g, m, nesterov=False)[0]
    for p in (-100, -60, 40, 120):
        assert torch.equal(step(w, g * 2.0 ** p, m, nesterov=False)[0], first), p


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_zeros_and_no_numbers(dtype):
    shape = (4, 40, 70)
    w, g, m = draw(shape, dtype, 10), draw(shape, dtype, 11), draw(shape, torch.float32, 12)
    clean = step(w, g, m)
    g[1], m[1] = 0.0, 0.0
    g[2, 5, 6] = float("inf")
    g[3, 39, 69] = float("nan")
    got = step(w, g, m)
    assert torch.equal(got[0][0], clean[0][0])                  # matrices of a stack do not meet
    assert torch.equal(got[0][1], (w[1].float() * (1 - 0.01)).to(dtype)) and not got[1][1].any()
    assert torch.isnan(got[0][2:]).all()
    assert torch.isinf(got[1][2]).sum() == 1 and torch.isnan(got[1][3]).sum() == 1


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_filters_of_a_layer_in_place_within_a_larger_array(dtype):
    """[LH][LW][K][F] as it is; nothing around it changes."""
    n = 3 * 5 * 48 * 20
    pad = 32
    rooms = [torch.full((n + 2 * pad,), 7.0, dtype=t, device="cuda") for t in (dtype, torch.float32)]
    w, m = (r[pad:pad + n].view(3, 5, 48, 20) for r in rooms)
    w.copy_(draw(w.shape, dtype, 13)), m.copy_(draw(w.shape, torch.float32, 14))
    g = draw(w.shape, dtype, 15)
    w0, m0 = w.clone().view(15, 48, 20), m.clone().view(15, 48, 20)
    lc.muon_step(w, g, m, None, None, 0.3, 0.01, 0.9, True, 5, code(dtype), scratch((15, 48, 20), dtype))
    check((w.view(15, 48, 20), m.view(15, 48, 20)), w0, g.view(15, 48, 20), m0)
    for r in rooms:
        assert (r[:pad] == 7).all() and (r[pad + n:] == 7).all()


def test_an_empty_stack():
    e = torch.empty(0, 5, 6, device="cuda")
    lc.muon_step(e, e, e, None, None, 0.1, ws=scratch((0, 5, 6), torch.float32))


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_captured_and_replayed(dtype):
    shape = (2, 130, 72)
    w, g, m = draw(shape, dtype, 16), draw(shape, dtype, 17), draw(shape, torch.float32, 18)
    wo, mo, ws = torch.empty_like(w), torch.empty_like(m), scratch(shape, dtype)

    def call():
        lc.muon_step(w, g, m, wo, mo, 0.2, 0.0, 0.9, True, 5, code(dtype), ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (19, 20, 21):
        g.copy_(draw(shape, dtype, seed))
        graph.replay()
        torch.cuda.synchronize()
        got = wo.clone(), mo.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], wo) and torch.equal(got[1], mo)


@pytest.mark.parametrize("dtype,shape", [(torch.float32, (1, 4291, 4291)), (torch.bfloat16, (9, 2436, 2436)), (torch.bfloat16, (2, 1024, 1024))], ids=str)
def test_large_square_matrices(shape, dtype):
    """Sides so long that a product with one costs more than two symmetric ones: no other order of products is taken, there is no shorter side."""
    print(f"case muon square {shape} {dtype}", flush=True)
    w, g, m = (torch.empty(shape, device="cuda").normal_(0, std, generator=torch.Generator("cuda").manual_seed(k)) for k, std in enumerate((0.5, 1.0, 4.0)))
    w, g = w.to(dtype), g.to(dtype)
    check(step(w, g, m), w, g, m, bounds=True)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 7])
@pytest.mark.parametrize("shape", [(1, 200, 2000), (1, 3000, 150), (2, 513, 4100), (9, 257, 300), (3, 512, 512), (40, 140, 130)], ids=str)
def test_groups_of_steps_and_small_tiles(shape, steps, dtype):
    """Sides beyond what one workgroup keeps: steps by groups and one by one, products in tiles of 32 and of more, sides that none of them divides."""
    print(f"case muon {shape} {steps} steps {dtype}", flush=True)
    w, g, m = draw(shape, dtype, 8, 2.0 ** -12), draw(shape, dtype, 9), draw(shape, torch.float32, 10, 4.0)
    got = step(w, g, m, steps=steps)
    check(got, w, g, m, steps=steps, bounds=True)
    again = step(w, g, m, steps=steps, in_place=True)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
