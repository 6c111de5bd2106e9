"""xent_fwd / xent_fwd_bwd against the definitions in 64 bits."""
import math

import pytest
import torch

import head_ref as ref
import paper_1502_03409_amd as lc

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (1, 64, 1000), (2, 7, 2), (5, 130, 77), (16, 64, 64), (17, 200, 129), (64, 96, 1025), (65, 257, 63), (130, 64, 500),
         (200, 100, 1333), (300, 520, 260)]


def dtypes(f):
    return pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])(f)


def code(dtype):
    return lc.LC_BF16 if dtype == torch.bfloat16 else lc.LC_F32


def inputs(N, D, V, dtype, seed=0, masked=0.25, std=2.0):
    gen = torch.Generator().manual_seed(seed)
    x, w = torch.randn((N, D), generator=gen), torch.randn((V, D), generator=gen) * std * D ** -0.5
    t = torch.randint(0, V, (N,), generator=gen)
    t[torch.rand(N, generator=gen) < masked] = -1
    return x.to(dtype).cuda(), w.to(dtype).cuda(), t.cuda()


def run(x, w, t, scale=None, grads=True, want_dx=True):
    (N, D), V = x.shape, w.shape[0]
    loss, cost = torch.full((N,), float("nan"), device="cuda"), torch.full((1,), float("nan"), device="cuda")
    nbytes = lc.xent_workspace_bytes(N, D, V, code(x.dtype), grads)
    ws = torch.full((nbytes // 4 + 64,), float("nan"), device="cuda")
    if not grads:
        lc.xent_fwd(x, w, t, scale, loss, cost, code(x.dtype), ws)
        return loss, cost
    dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    lc.xent_fwd_bwd(x, w, t, scale, loss, cost, dx if want_dx else None, dw, code(x.dtype), ws)
    return loss, cost, dx, dw


def loss_bound(x, w):
    """A score is off by at most its fp32 sum's error; the loss by twice that, and by 2^-20 for the exponentials, the logarithm and
    the joining of tiles, all absolute."""
    D = x.shape[1]
    worst = float((x.double().abs() @ w.double().abs().t()).nan_to_num(0, 0, 0).max()) if x.shape[0] else 0.0
    return 2 * 2.0 ** -24 * (math.sqrt(6 * D) + 4) * worst + 2.0 ** -20


def check_all(x, w, t, scale, got):
    loss, cost, dx, dw = got
    rl, rc, rx, rw = ref.xent(x, w, t, scale)
    live = torch.where((t >= 0)[:, None], x.float(), 0.0)
    b = loss_bound(live, w)
    assert float((loss.double() - rl).abs().max()) <= b + 2.0 ** -23 * float(rl.abs().max())
    s = scale if scale is not None else torch.full_like(loss, 1.0 / max(1, int((t >= 0).sum())))
    total = float((s.double().abs() * (t >= 0)).sum())
    assert abs(float(cost) - float(rc)) <= total * b + 2.0 ** -22 * abs(float(rc))
    # a probability is off by the scores' error; roundings to bf16: d and the result's own (the exponential's are an eighth of one)
    bound = ref.tol(x.dtype, max(x.shape[0], w.shape[0]), 2.25) + b
    ref.check("dx", dx, rx, bound)
    ref.check("dw", dw, rw, bound)


@dtypes
@pytest.mark.parametrize("N,D,V", SIZES)
def test_values_and_gradients(N, D, V, dtype):
    print(f"case xent {N} {D} {V} {dtype}", flush=True)
    x, w, t = inputs(N, D, V, dtype)
    if N > 1:
        t[N - 1], t[0] = V - 1, 0       # the last word, the first, and at least these rows
    got = run(x, w, t)
    check_all(x, w, t, None, got)
    loss, cost = run(x, w, t, grads=False)
    assert torch.equal(loss, got[0]) and torch.equal(cost, got[1])
    _, _, _, dw = run(x, w, t, want_dx=False)
    assert torch.equal(dw, got[3])


@dtypes
def test_weights_of_rows(dtype):
    x, w, t = inputs(90, 70, 300, dtype, seed=1)
    scale = torch.rand(90, generator=torch.Generator().manual_seed(2)).cuda()
    scale[t < 0] = float("nan")      # not looked at
    scale[5] = 0.0
    got = run(x, w, t, scale)
    check_all(x, w, t, torch.where(t >= 0, scale, 0.0), got)


@dtypes
@pytest.mark.parametrize("N", [0, 1, 70])
def test_no_row_left(N, dtype):
    x, w, t = inputs(N, 33, 40, dtype)
    t.fill_(-1)
    x.fill_(float("nan"))
    loss, cost, dx, dw = run(x, w, t)
    assert not loss.any() and float(cost) == 0.0 and not dx.any() and not dw.any()
    loss, cost = run(x, w, t, grads=False)
    assert not loss.any() and float(cost) == 0.0


@dtypes
def test_masked_rows_are_not_looked_at(dtype):
    x, w, t = inputs(150, 70, 260, dtype, seed=3, masked=0.5)
    clean = run(x, w, t)
    x2 = x.clone()
    x2[t < 0] = float("nan")
    x2[torch.nonzero(t < 0)[0]] = float("inf")
    t2 = torch.where(t < 0, torch.full_like(t, -(1 << 40)), t)      # any negative number masks
    for a, b in zip(clean, run(x2, w, t2)):
        assert torch.equal(a, b)


@dtypes
def test_a_target_outside_the_vocabulary_is_loud(dtype):
    x, w, t = inputs(20, 40, 100, dtype, masked=0.0)
    t[7] = 100
    t[8] = 1 << 40
    loss, cost, dx, dw = run(x, w, t)
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[7] = bad[8] = True
    assert torch.equal(torch.isnan(loss), bad) and torch.isnan(cost).all()
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all() and torch.isnan(dw).all()


@dtypes
def test_rows_that_are_learned_keep_small_gradients(dtype):
    """Scores far apart: the target's probability is 1 - 10^-6 or so, and the gradient is made of what is left."""
    gen = torch.Generator().manual_seed(7)
    N, D, V = 40, 64, 200
    w = torch.randn((V, D), generator=gen).to(dtype)
    t = torch.randint(0, V, (N,), generator=gen)
    x = (w[t].float() * 0.4 + 0.05 * torch.randn((N, D), generator=gen)).to(dtype)
    x, w, t = x.cuda(), w.cuda(), t.cuda()
    _, _, rx, rw = ref.xent(x, w, t)
    _, _, dx, dw = run(x, w, t)
    # p and p - 1 are relative to the scores' error, which is absolute
    bound = ref.tol(dtype, V, 2.25) + loss_bound(x.float(), w)
    ref.check("dx", dx, rx, bound)
    ref.check("dw", dw, rw, bound)


@dtypes
def test_scores_of_any_size(dtype):
    """Differences of thousands between scores; a word that no row can reach (its scores are -inf) changes nothing else."""
    x, w, t = inputs(50, 32, 150, dtype, seed=8, masked=0.1, std=3000.0)
    loss, cost, dx, dw = run(x, w, t)
    rl, rc, rx, rw = ref.xent(x, w, t)
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    b = loss_bound(x.float(), w)
    assert float((loss.double() - rl).abs().max()) <= b + 2.0 ** -23 * float(rl.abs().max())
    x, w, t = inputs(20, 32, 150, dtype, seed=9, masked=0.0)
    x[:, 0] = 1.0
    w[77] = 0.0
    w[77, 0] = float("-inf")
    t[t == 77] = 0
    loss, cost = run(x, w, t, grads=False)
    keep = torch.arange(150, device="cuda") != 77
    rl, rc, _, _ = ref.xent(x, w[keep], torch.where(t > 77, t - 1, t))
    assert float((loss.double() - rl).abs().max()) <= loss_bound(x.float(), w[keep])


def test_gradients_against_differences():
    x, w, t = inputs(40, 60, 90, torch.float32, seed=10)
    scale = torch.rand(40, generator=torch.Generator().manual_seed(2)).cuda()
    _, _, dx, dw = run(x, w, t, scale)
    gen = torch.Generator().manual_seed(5)
    ex, ew = (torch.randn(a.shape, generator=gen, dtype=torch.float64).cuda() for a in (x, w))

    def cost(e):
        return float(ref.xent(x.double() + e * ex, w.double() + e * ew, t, scale)[1])

    quotient = (cost(1e-5) - cost(-1e-5)) / 2e-5
    inner = float((dx.double() * ex).sum() + (dw.double() * ew).sum())
    size = float(dx.double().norm() * ex.norm() + dw.double().norm() * ew.norm())
    assert abs(inner - quotient) <= (ref.tol(torch.float32, 90, 0) + loss_bound(x, w)) * size


@pytest.mark.parametrize("dtype,N,V", [(torch.bfloat16, 6000, 200001), (torch.float32, 3100, 200001)], ids=["bf16", "f32"])
def test_more_rows_than_are_kept_at_a_time(dtype, N, V):
    """The exponentials of all rows exceed what is kept at once: the weight gradient adds up over blocks of rows."""
    D = 72
    print(f"case xent blocks {N} {D} {V} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((N, D), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((V, D), generator=gen, device="cuda") * 2 * D ** -0.5).to(dtype)
    t = torch.randint(0, V, (N,), generator=gen, device="cuda")
    t[torch.rand(N, generator=gen, device="cuda") < 0.1] = -1
    loss, cost, dx, dw = run(x, w, t)
    rx, rw, rl = torch.empty(N, D, device="cuda", dtype=torch.float64), torch.zeros(V, D, device="cuda", dtype=torch.float64), []
    count = int((t >= 0).sum())
    for i in range(0, N, 1000):
        s = torch.full((min(1000, N - i),), 1.0 / count, device="cuda")
        l, _, a, b = ref.xent(x[i:i + 1000], w, t[i:i + 1000], s)
        rl.append(l)
        rx[i:i + 1000] = a
        rw += b
    b = loss_bound(x.float(), w)
    assert float((loss.double() - torch.cat(rl)).abs().max()) <= b
    bound = ref.tol(dtype, V, 2.25) + b
    ref.check("dx", dx, rx, bound)
    ref.check("dw", dw, rw, bound)


@dtypes
def test_the_same_bits_on_another_stream_and_in_a_graph(dtype):
    x, w, t = inputs(130, 100, 700, dtype, seed=11)
    first = run(x, w, t)
    (N, D), V = x.shape, w.shape[0]
    loss, cost, dx, dw = (torch.empty_like(a) for a in first)
    ws = torch.empty(lc.xent_workspace_bytes(N, D, V, code(dtype), True), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lc.xent_fwd_bwd(x, w, t, None, loss, cost, dx, dw, code(dtype), ws)
    side.synchronize()
    for a, b in zip(first, (loss, cost, dx, dw)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lc.xent_fwd_bwd(x, w, t, None, loss, cost, dx, dw, code(dtype), ws)
    for _ in range(3):
        ws.fill_(255)
        for a in (loss, cost, dx, dw):
            a.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(first, (loss, cost, dx, dw)):
            assert torch.equal(a, b)


@dtypes
@pytest.mark.parametrize("N", [5, 70])
def test_a_row_whose_scores_are_all_minus_infinity_is_loud(N, dtype):
    """The logarithm of nothing less the logarithm of nothing: NaN, for one word and for many."""
    for V in (1, 150):
        x, w, t = inputs(N, 33, V, dtype, seed=12, masked=0.0)
        x[:, 0] = 1.0
        w[:, 0] = float("-inf")
        t[1] = -1
        live = t >= 0
        for grads in (False, True):
            loss, cost = run(x, w, t, grads=grads)[:2]
            assert torch.equal(torch.isnan(loss), live) and torch.isnan(cost).all()


@dtypes
@pytest.mark.parametrize("low", [-1e5, float("-inf")])
@pytest.mark.parametrize("N", [5, 70])
def test_a_target_far_below_the_other_words(N, low, dtype):
    """The other words' probabilities are as exact as their own scores.  The target's score is `low`, its gradient -1 times the row's
    weight; the cost of an impossible target is infinite, its gradients by words are finite."""
    x, w, t = inputs(N, 33, 150, dtype, seed=13, masked=0.1)
    x[:, 0] = 1.0
    w[:, 0] = 0.0
    w[77] = 0.0
    w[77, 0] = low
    t[0], t[3], t[4] = 77, 77, 78
    loss, cost, dx, dw = run(x, w, t)
    rl, rc, rx, rw = ref.xent(x, w, t)
    others = torch.arange(150, device="cuda") != 77
    b = loss_bound(x.float(), w[others])
    impossible = torch.isinf(rl)
    assert torch.equal(torch.isinf(loss), impossible) and bool((impossible == ((t == 77) & (low < -1e30))).all())
    near = ~impossible
    assert float((loss.double() - rl)[near].abs().max()) <= b + 2.0 ** -23 * float(rl[near].abs().max())
    assert torch.isinf(cost).all() if low < -1e30 else abs(float(cost) - float(rc)) <= b + 2.0 ** -22 * float(rc)
    bound = ref.tol(dtype, N, 2.25) + b
    ref.check("dw", dw[others], rw[others], bound)
    ref.check("dw of the target", dw[77], rw[77], bound)
    live = t >= 0      # a masked row's dx is zero, whatever the words are
    ref.check("dx", dx[live], rx[live], ref.tol(dtype, 150, 2.25) + b)
    assert not dx[~live].any()


def check_equal_scores(N, dtype, size):
    """Half of the words share the score `size`, up to the row's sign, the others have its half: one product each, so all scores are
    exact, and the probabilities are those of a draw among the largest."""
    x = torch.full((N, 1), size, device="cuda").to(dtype)
    x[1::2] *= -1
    w = torch.ones((150, 1), device="cuda").to(dtype)
    w[::2] = 0.5
    t = torch.arange(N, device="cuda") * 2 % 150 + (torch.arange(N, device="cuda") + 1) % 2      # among the largest
    t[2] = -1
    loss, cost, dx, dw = run(x, w, t)
    live = t >= 0
    # the exponentials, their sum and its logarithm
    bound = 2.0 ** -20 * math.log(75)
    assert float((loss.double() - math.log(75) * live).abs().max()) <= bound
    assert abs(float(cost) - math.log(75)) <= bound
    d = torch.zeros((N, 150), dtype=torch.float64, device="cuda")
    d[0::2, 1::2] = d[1::2, 0::2] = 1 / 75
    d.scatter_add_(1, t.clamp(min=0)[:, None], torch.full((N, 1), -1.0, dtype=torch.float64, device="cuda"))
    d = d * live[:, None] / int(live.sum())
    # a word's gradient adds up terms of size * p of either sign: its bound is that of the sum of their magnitudes, of which it is a part
    want, total = d.t() @ x.double(), d.abs().t() @ x.double().abs()
    assert bool(((dw.double() - want).abs() <= (ref.tol(dtype, N, 2.25) + bound) * total).all())
    assert torch.isfinite(dx).all() and not dx[~live].any()


@pytest.mark.parametrize("size", [1e4, 1e8, 1e30, 1e38])
@pytest.mark.parametrize("N", [5, 70])
def test_equal_scores_of_any_size(N, size):
    check_equal_scores(N, torch.float32, size)


@pytest.mark.parametrize("size", [1e4, 1e8, 1e30, 1e38])
@pytest.mark.parametrize("N", [5, 70])
def test_equal_scores_of_any_size_in_bf16(N, size):
    check_equal_scores(N, torch.bfloat16, size)


@dtypes
@pytest.mark.parametrize("N", [5, 70])
def test_words_that_hardly_count_have_their_gradients(N, dtype):
    """Words whose scores lie 30 to 60 below the largest, beside it in a tile and in tiles of their own: probabilities down to 10^-26 are
    as exact as others, relative to their own size.  One product a score, so the scores' rounding is that of their size."""
    gen = torch.Generator().manual_seed(14)
    V = 300
    x = (1.0 + 0.1 * torch.rand(N, 1, generator=gen)).to(dtype).cuda()
    w = (-30.0 - 25.0 * torch.rand(V, 1, generator=gen)).to(dtype).cuda()
    w[5] = 0.0
    t = torch.full((N,), 5, device="cuda")
    t[1] = -1
    loss, cost, dx, dw = run(x, w, t)
    _, _, rx, rw = ref.xent(x, w, t)
    others = torch.arange(V, device="cuda") != 5
    bound = ref.tol(dtype, N, 2.25) + 4 * 2.0 ** -24 * 60
    worst = float(((dw.double() - rw).abs() / rw.abs())[others].max())
    assert worst <= bound, (worst, bound)
    ref.check("dx", dx, rx, bound)


@dtypes
@pytest.mark.parametrize("N", [5, 70])
def test_gradients_of_scores_far_apart(N, dtype):
    """Two groups of words 3000 apart, each with a spread of a few: one product a score, so scores are exact and probabilities those of
    the upper group, which is another for rows of the other sign."""
    gen = torch.Generator().manual_seed(15)
    x = torch.ones(N, 1)
    x[1::2] = -1
    w = torch.randn(150, 1, generator=gen) * 2 + 3000 * (torch.rand(150, 1, generator=gen) < 0.5)
    t = torch.randint(0, 150, (N,), generator=gen)
    t[2] = -1
    x, w, t = x.to(dtype).cuda(), w.to(dtype).cuda(), t.cuda()
    loss, cost, dx, dw = run(x, w, t)
    rl, rc, rx, rw = ref.xent(x, w, t)
    # the loss is rounded at its own size, the differences of scores within a group at theirs (below 64)
    assert bool(((loss.double() - rl).abs() <= 2.0 ** -20 + 2.0 ** -22 * rl).all())
    assert abs(float(cost) - float(rc)) <= 2.0 ** -20 + 2.0 ** -22 * float(rc)
    bound = ref.tol(dtype, N, 2.25) + 4 * 2.0 ** -24 * 64
    ref.check("dw", dw, rw, bound)
    # dx adds up 150 words of up to 3000 with weights of either sign: its bound is that of the sum of magnitudes
    live = t >= 0
    d = torch.softmax(x.double() @ w.double().t(), dim=1) + torch.nn.functional.one_hot(t.clamp(min=0), 150)
    total = d @ w.double().abs() / int(live.sum())
    assert bool(((dx.double() - rx).abs() <= (ref.tol(dtype, 150, 2.25) + 4 * 2.0 ** -24 * 64) * total)[live].all())
    assert not dx[~live].any()


@dtypes
@pytest.mark.parametrize("N", [1, 2, 9, 32])
@pytest.mark.parametrize("masked", [0.0, 0.5])
def test_weights_of_few_rows_are_not_rounded(N, masked, dtype):
    """Rows with a weight half way between two bf16 numbers, the same for all: rounded to either, all gradients were 0.4 % too short or too
    long.  Against the exact gradient, rounded once: what is off along it is what was off before that rounding, 2^-16 for d in two
    parts and less for the probabilities' 2^-10 (a hundredth of the gradients' squares).  Results are a number times one of the 128 significands
    that bf16 has, so those that cross from one bf16 number to the next do so a 128th, or 2^-15 of the gradient, at a time: 2^-11 is sixteen."""
    D, V = 2000, 250
    x, w, t = inputs(N, D, V, dtype, seed=16, masked=masked, std=0.5)
    t[0] = 7
    scale = torch.full((N,), 1.00390625, device="cuda")
    loss, cost, dx, dw = run(x, w, t, scale)
    rl, rc, rx, rw = ref.xent(x, w, t, torch.where(t >= 0, scale, 0.0))
    for got, want in ((dx, rx), (dw, rw)):
        along = float(((got.double() - want.to(dtype).double()) * want).sum() / (want * want).sum())
        assert abs(along) <= (2.0 ** -11 if dtype == torch.bfloat16 else ref.tol(dtype, D, 0)), along
    check_all(x, w, t, torch.where(t >= 0, scale, 0.0), (loss, cost, dx, dw))
    assert not dx[t < 0].any()
