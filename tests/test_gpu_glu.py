"""glu_fwd / glu_bwd against the definitions in 64 bits."""
import numpy
import pytest
import torch

import head_ref as ref
import paper_1502_03409_amd as lc

pytestmark = pytest.mark.gpu

CODE = {"sigmoid": lc.LC_ACT_SIGMOID, "silu": lc.LC_ACT_SILU, "gelu": lc.LC_ACT_GELU}
SIZES = [(1, 1, 1), (1, 64, 64), (2, 8, 200), (3, 65, 33), (16, 256, 96), (17, 200, 130), (33, 130, 31), (64, 64, 32), (70, 320, 260),
         (129, 257, 65), (200, 1000, 300), (257, 512, 513), (300, 72, 1100)]


def dtypes(f):
    return pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])(f)


def code(dtype):
    return lc.LC_BF16 if dtype == torch.bfloat16 else lc.LC_F32


def inputs(N, D, F, dtype, seed=0, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    x, wg, wu, dh = (torch.randn(s, generator=gen) for s in ((N, D), (F, D), (F, D), (N, F)))
    return tuple(t.to(dtype).cuda() for t in (x * std, wg * D ** -0.5, wu * D ** -0.5, dh / N))


def scratch(nbytes):
    return torch.full((nbytes // 4 + 64,), float("nan"), device="cuda")


def saved(codes):
    """The values of a 16-bit code of g or u (fp32: the values themselves)."""
    if codes.dtype == torch.float32:
        return codes.double()
    c = codes.contiguous().view(torch.int16).int() & 0xffff
    bits = torch.where((c & 0x4000) != 0, (c & 0x3fff) << 17, ((c & 0x3fff) << 14) + (111 << 23))
    return (bits | ((c >> 15) << 31)).view(torch.float32).double()


def forward(x, wg, wu, name, save=True, ws=None):
    (N, D), F = x.shape, wg.shape[0]
    h = torch.full((N, F), float("nan"), dtype=x.dtype, device="cuda")
    gu = torch.full((N, 2, F), float("nan"), dtype=x.dtype, device="cuda") if save else None
    ws = scratch(lc.glu_workspace_bytes(N, D, F, code(x.dtype))) if ws is None else ws
    lc.glu_fwd(x, wg, wu, h, gu, CODE[name], code(x.dtype), ws)
    return h, gu


def backward(x, wg, wu, gu, dh, name, want_dx=True):
    (N, D), F = x.shape, wg.shape[0]
    out = [torch.full_like(t, float("nan")) for t in (x, wg, wu)]
    ws = scratch(lc.glu_workspace_bytes(N, D, F, code(x.dtype), True))
    lc.glu_bwd(x, wg, wu, gu, dh, out[0] if want_dx else None, out[1], out[2], CODE[name], code(x.dtype), ws)
    return out


@dtypes
@pytest.mark.parametrize("name", ref.ACTS)
@pytest.mark.parametrize("N,D,F", SIZES)
def test_values_and_gradients(N, D, F, name, dtype):
    print(f"case glu {N} {D} {F} {name} {dtype}", flush=True)
    x, wg, wu, dh = inputs(N, D, F, dtype)
    h, gu = forward(x, wg, wu, name)
    rh, rg, ru = ref.glu(x, wg, wu, name)
    ref.check("h", h, rh, ref.tol(dtype, D, 1))
    for k, r in ((0, rg), (1, ru)):
        ref.check("gu", saved(gu[:, k]), r, ref.tol(dtype, D, 0) + (2.0 ** -10 if dtype == torch.bfloat16 else 0.0))
    h2, _ = forward(x, wg, wu, name, save=False)
    assert torch.equal(h, h2)
    dx, dwg, dwu = backward(x, wg, wu, gu, dh, name)
    rx, rwg, rwu = ref.glu_grads(x, wg, wu, dh, name)
    # roundings to bf16: dg and the result's own; those of g (whose derivative act' follows within a factor of two) and u are a
    # quarter of one each
    ref.check("dx", dx, rx, ref.tol(dtype, D + 2 * F, 2.75))
    ref.check("dwg", dwg, rwg, ref.tol(dtype, D + N, 2.75))
    ref.check("dwu", dwu, rwu, ref.tol(dtype, D + N, 2.75))
    _, dwg2, dwu2 = backward(x, wg, wu, gu, dh, name, want_dx=False)
    assert torch.equal(dwg, dwg2) and torch.equal(dwu, dwu2)


@pytest.mark.parametrize("name", ref.ACTS)
def test_gradients_against_differences(name):
    """Along a random direction of all three inputs: the kernels' gradients against the difference quotient of the cost in 64
    bits.  With steps of 1e-5 the quotient is good to 1e-9; the gradients are held to their own bound, times the ratio of the norms
    that a single inner product can lose."""
    x, wg, wu, dh = inputs(40, 100, 70, torch.float32, seed=3)
    _, gu = forward(x, wg, wu, name)
    grads = backward(x, wg, wu, gu, dh, name)
    gen = torch.Generator().manual_seed(5)
    dirs = [torch.randn(t.shape, generator=gen, dtype=torch.float64).cuda() for t in (x, wg, wu)]

    def cost(e):
        h, _, _ = ref.glu(*(t.double() + e * d for t, d in zip((x, wg, wu), dirs)), name)
        return float((h * dh.double()).sum())

    quotient = (cost(1e-5) - cost(-1e-5)) / 2e-5
    inner = sum(float((g.double() * d).sum()) for g, d in zip(grads, dirs))
    size = sum(float(g.double().norm() * d.norm()) for g, d in zip(grads, dirs))
    assert abs(inner - quotient) <= ref.tol(torch.float32, 240, 0) * size


@dtypes
def test_no_rows(dtype):
    x, wg, wu, dh = inputs(0, 40, 24, dtype)[0], *inputs(1, 40, 24, dtype)[1:3], torch.empty(0, 24, dtype=dtype, device="cuda")
    h, gu = forward(x, wg, wu, "silu")
    assert h.shape == (0, 24)
    _, dwg, dwu = backward(x, wg, wu, gu, dh, "silu")
    assert not dwg.any() and not dwu.any()


@dtypes
def test_infinities_and_nan_stay_in_their_rows(dtype):
    x, wg, wu, _ = inputs(70, 96, 64, dtype, seed=2)
    x[3, 5], x[40, 7], x[69, 0] = float("inf"), float("nan"), float("-inf")
    h, _ = forward(x, wg, wu, "silu")
    rh, rg, ru = ref.glu(x, wg, wu, "silu")
    bad = torch.zeros(70, dtype=torch.bool)
    bad[[3, 40, 69]] = True
    ref.check("other rows", h[~bad.cuda()], rh[~bad.cuda()], ref.tol(dtype, 96, 1))
    _, gu = forward(x, wg, wu, "silu")
    for k, r in ((0, rg), (1, ru)):      # a single infinite factor: infinities of the right sign, NaN where NaN went in
        ref.check("projections", saved(gu[:, k]), r, ref.tol(dtype, 96, 1))


def test_the_code_of_saved_values():
    """Through a layer of one weight (g = u = x): ten bits between 2^-16 and 2^16, seven elsewhere, signs, infinities, NaN, zero."""
    gen = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(3000, generator=gen) * 2.0 ** k for k in (-120, -40, -17, -15, -1, 0, 5, 15, 17, 60, 120)])
    x = torch.cat([x, torch.tensor([0.0, float("inf"), float("-inf"), float("nan"), 65535.9, 65536.0, 2.0 ** -16, 3.4e38, 1e-39])])
    x = x.bfloat16()[:, None].cuda()
    w = torch.full((1, 1), 1.00390625, device="cuda").bfloat16() * 1.0078125      # products need more than eight bits
    _, gu = forward(x, w, w, "silu")
    want = (x.double() * w.double())[:, 0].float()
    got = saved(gu[:, 0, 0])
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    near = fine & (want.abs() >= 2.0 ** -16) & (want.abs() < 65536.0 * (1 - 2.0 ** -11))
    assert bool(((got - want.double()).abs()[near] <= 2.0 ** -10 * want.double().abs()[near]).all())
    far = fine & ~near & (want.abs() < 3e38)
    assert bool(((got - want.double()).abs()[far] <= 2.0 ** -7 * want.double().abs()[far] + 2.0 ** -132).all())
    inf = torch.isinf(want)
    assert torch.equal(got[inf].float(), want[inf]) and bool((got[far].sign() * want[far].sign() >= 0).all())
    assert torch.equal(gu[:, 0].contiguous().view(torch.int16), gu[:, 1].contiguous().view(torch.int16))


@pytest.mark.parametrize("N", [5, 150])
def test_saved_values_bit_by_bit(N):
    """Neighbouring outputs on both sides of the marked form's border, in kernels for few rows and in tiles.  Products of two bf16
    numbers are exact in fp32, so the code of each is known."""
    gen = torch.Generator().manual_seed(7)
    F = 150
    x = torch.randn(N, 1, generator=gen).bfloat16()
    x[1] = 0
    x[2, 0], x[3, 0], x[4, 0] = float("inf"), float("nan"), -0.0
    exponent = torch.randint(-40, 40, (F, 1), generator=gen) * (torch.rand(F, 1, generator=gen) < 0.3)
    w = (torch.randn(F, 1, generator=gen) * 2.0 ** exponent).bfloat16()
    x[0, 0] = 1
    w[:6, 0] = torch.tensor([65280.0, 65536.0, 2.0 ** -16, 2.0 ** -17, 1.9921875 * 2.0 ** 15, -1.9921875 * 2.0 ** -17])
    v = (x.float() * w.float().T).numpy().view("uint32").astype("int64")
    sign, mag = (v >> 16) & 0x8000, v & 0x7FFFFFFF
    near = ((mag + 0x1FFF + ((mag >> 14) & 1)) >> 14) - (111 << 9)
    far = (mag + 0xFFFF + ((mag >> 17) & 1)) >> 17
    nan = mag > 0x7F800000
    want = sign | numpy.where((near >= 0) & (near < 32 << 9), near, 0x4000 | far)
    _, gu = forward(x.cuda(), w.cuda(), w.cuda(), "sigmoid")
    for k in (0, 1):
        got = gu[:, k].cpu().contiguous().view(torch.int16).numpy().astype("int64") & 0xFFFF
        assert (got[~nan] == want[~nan])[mag[~nan] != 0].all()
        assert ((got[~nan] & 0x7FFF) == (want[~nan] & 0x7FFF)).all()      # a zero may lose its sign in a sum
        assert ((got[nan] & 0x7FE0) == 0x7FE0).all()


def test_small_and_large_fp32_operands():
    """Operands at the ends of the exponent range: bits of 2^-133 and above count, so an operand is off by 2^-134 at most; sums that
    overflow before they come back never become NaN."""
    for std in (1e-33, 1e-37, 3e-41, 1e30):
        x, wg, wu, _ = inputs(20, 70, 40, torch.float32, seed=4, std=std)
        _, gu = forward(x, wg, wu, "sigmoid")
        _, rg, ru = ref.glu(x, wg, wu, "sigmoid")
        bound = ref.tol(torch.float32, 70, 0) + (2.0 ** -134 + 2.0 ** -149 * 70) / std
        ref.check(f"g {std}", gu[:, 0], rg, bound)
        ref.check(f"u {std}", gu[:, 1], ru, bound)
    x = torch.full((3, 4), 3e38, device="cuda")
    w = torch.tensor([[1.0, 1.0, -1.0, -0.5]], device="cuda")
    _, gu = forward(x, w, w, "sigmoid")
    assert not torch.isnan(gu).any()


@dtypes
def test_the_same_bits_every_time_on_any_stream(dtype):
    x, wg, wu, dh = inputs(150, 200, 170, dtype, seed=6)
    first = forward(x, wg, wu, "gelu")
    gfirst = backward(x, wg, wu, first[1], dh, "gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = forward(x, wg, wu, "gelu")
        gagain = backward(x, wg, wu, again[1], dh, "gelu")
    side.synchronize()
    for a, b in zip((*first, *gfirst), (*again, *gagain)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("N", [3, 100])
def test_large_saved_values_stay_finite(N):
    """The largest numbers of bf16 lie above the largest seven bits: they are saved as that, not as infinities, which times a
    gradient of zero would be NaN."""
    x = torch.full((N, 1), torch.finfo(torch.bfloat16).max, dtype=torch.bfloat16, device="cuda")
    x[1] *= -1
    w = torch.ones((9, 1), dtype=torch.bfloat16, device="cuda")
    _, gu = forward(x, w, w, "sigmoid")
    want = x.double().expand(N, 9)
    for k in (0, 1):
        assert bool(((saved(gu[:, k]) - want).abs() <= 2.0 ** -7 * want.abs()).all())
    for grad in backward(x, w, w, gu, torch.zeros((N, 9), dtype=torch.bfloat16, device="cuda"), "sigmoid"):
        assert not grad.any()


@dtypes
@pytest.mark.parametrize("name", ["sigmoid", "silu"])
def test_gates_that_are_open_wide_or_shut(name, dtype):
    """The gate's derivative by itself (one row, x = u = dh = 1), relative to its own size: e^-|g| however small.  Gates in steps of 1/4
    up to 16 are exact in every type on the way."""
    g = torch.arange(-64, 65, device="cuda")[:, None] / 4
    x, wg, wu, dh = (t.to(dtype) for t in (torch.ones((1, 1), device="cuda"), g, torch.ones_like(g), torch.ones((1, 129), device="cuda")))
    _, gu = forward(x, wg, wu, name)
    _, dwg, dwu = backward(x, wg, wu, gu, dh, name)
    a, da = ref.act(name, g.double())
    rest = torch.sigmoid(-g.double())
    da = a * rest if name == "sigmoid" else torch.sigmoid(g.double()) * (1 + g * rest)
    # SiLU's derivative crosses zero, as a sum of one and g (1 - s): an error of one rounding of the larger of both
    size = da.abs() if name == "sigmoid" else torch.sigmoid(g.double()) * torch.maximum(torch.ones_like(g), (g * rest).abs())
    assert bool(((dwg.double() - da).abs() <= ref.tol(dtype, 1, 2.75) * size).all())
    assert bool(((dwu.double() - a).abs() <= ref.tol(dtype, 1, 2.75) * a.abs()).all())


@dtypes
@pytest.mark.parametrize("N", [1, 2, 9, 32])
def test_gradients_of_few_rows_are_not_rounded(N, dtype):
    """All dg the same and half way between two bf16 numbers (u = 3/2, dh = 1 + 2^-7, act' = 1/4): rounded to either, the gradient of wg
    was 0.26 % too short or too long.  Against the exact gradient, rounded once; the bound is that of 16 crossings of one significand of
    128 from one bf16 number to the next, each 2^-15 of the gradient, where 2^-16 of it is left of d in two parts."""
    D, F = 2000, 70
    gen = torch.Generator().manual_seed(8)
    x = torch.randn(N, D, generator=gen)
    x[:, 0] = 1.0
    wg, wu = torch.zeros(F, D), torch.zeros(F, D)
    wu[:, 0] = 1.5
    dh = torch.full((N, F), 1.0078125)
    x, wg, wu, dh = (t.to(dtype).cuda() for t in (x, wg, wu, dh))
    _, gu = forward(x, wg, wu, "sigmoid")
    dx, dwg, dwu = backward(x, wg, wu, gu, dh, "sigmoid")
    rx, rwg, rwu = ref.glu_grads(x, wg, wu, dh, "sigmoid")
    for what, got, want in (("dwg", dwg, rwg), ("dwu", dwu, rwu)):
        along = float(((got.double() - want.to(dtype).double()) * want).sum() / (want * want).sum())
        assert abs(along) <= (2.0 ** -11 if dtype == torch.bfloat16 else ref.tol(dtype, D, 0)), (what, along)
    ref.check("dx", dx, rx, ref.tol(dtype, D + 2 * F, 2.75))


@dtypes
@pytest.mark.parametrize("N", [3, 32, 33])
def test_infinities_in_gradients_of_few_rows(N, dtype):
    """An infinite feature, an infinite weight and an infinite gradient: infinities and NaN where the formulas have them, nothing else."""
    x, wg, wu, dh = inputs(N, 96, 200, dtype, seed=9)
    _, gu = forward(x, wg, wu, "silu")
    x[1, 11], wg[3, 5], dh[2, 7] = float("inf"), float("-inf"), float("inf")
    dx, dwg, dwu = backward(x, wg, wu, gu, dh, "silu")
    g, u = saved(gu[:, 0]), saved(gu[:, 1])
    a, da = ref.act("silu", g)
    dg, du = dh.double() * u * da, dh.double() * a
    bound = ref.tol(dtype, 500, 2.75)
    ref.check("dx", dx, dg @ wg.double() + du @ wu.double(), bound)
    ref.check("dwg", dwg, dg.t() @ x.double(), bound)
    ref.check("dwu", dwu, du.t() @ x.double(), bound)
