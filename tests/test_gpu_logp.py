"""logp_fwd / logp_bwd against the definitions in 64 bits."""
import math

import pytest
import torch

import head_ref as ref
import paper_1502_03409_amd as lc

pytestmark = pytest.mark.gpu

# one row to tiles of 128 and 256, words around 32, 64, 128 and one
SIZES = [(1, 1, 1, 0, 1), (1, 64, 1000, 0, 10), (2, 7, 2, 1, 2), (5, 130, 77, 3, 64), (16, 64, 64, 2, 33), (17, 200, 129, 16, 1), (32, 96, 1025, 0, 5),
         (33, 40, 31, 1, 31), (64, 96, 1025, 1, 40), (65, 257, 63, 2, 0), (130, 64, 500, 0, 20), (200, 100, 1333, 5, 7), (300, 520, 260, 64, 64)]


def dtypes(f):
    return pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])(f)


def code(dtype):
    return lc.LC_BF16 if dtype == torch.bfloat16 else lc.LC_F32


def inputs(N, D, V, T, dtype, seed=0, masked=0.25, std=2.0):
    gen = torch.Generator().manual_seed(seed)
    x, w = torch.randn((N, D), generator=gen), torch.randn((V, D), generator=gen) * std * D ** -0.5
    x = x * (0.2 + 1.6 * torch.rand((N, 1), generator=gen))
    t = torch.randint(0, V, (N, T), generator=gen)
    t[torch.rand((N, T), generator=gen) < 0.3] = -1
    t[torch.rand(N, generator=gen) < masked] = -5
    if T and N > 1:
        t[0], t[N - 1, 0] = 0, V - 1       # a row of the same word, and at least these rows
    return x.to(dtype).cuda(), w.to(dtype).cuda(), t.cuda() if T else None


def blank(shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), device="cuda").to(dtype) if dtype.is_floating_point else torch.full(shape, -77, dtype=dtype, device="cuda")


def scratch(N, D, V, T, K, dtype, grads):
    return torch.full((lc.logp_workspace_bytes(N, D, V, T, K, code(dtype), grads) // 4 + 64,), float("nan"), device="cuda")


def answers(x, w, tags, K, entropy=True, state=True):
    (N, D), V, T = x.shape, w.shape[0], 0 if tags is None else tags.shape[1]
    out = {"logp": blank((N, T)) if T else None, "entropy": blank((N,)) if entropy else None, "top": blank((N, K), torch.int64) if K else None,
           "top_logp": blank((N, K)) if K else None, "state": blank((N, 3)) if state else None}
    lc.logp_fwd(x, w, tags, out["logp"], out["entropy"], out["top"], out["top_logp"], out["state"], code(x.dtype),
                scratch(N, D, V, T, K, x.dtype, False))
    return out


def gradients(x, w, tags, got, dlogp, dentropy, want_dx=True):
    (N, D), V, T = x.shape, w.shape[0], 0 if tags is None else tags.shape[1]
    dx, dw = blank(x.shape, x.dtype) if want_dx else None, blank(w.shape, w.dtype)
    lc.logp_bwd(x, w, tags, got["logp"], got["state"], dlogp, dentropy, dx, dw, code(x.dtype), scratch(N, D, V, T, 0, x.dtype, True))
    return dx, dw


def definition(x, w, tags, K):
    live = (tags >= 0).any(dim=1) if tags is not None else torch.ones(x.shape[0], dtype=torch.bool, device="cuda")
    xd, wd = torch.where(live[:, None], x.double(), 0.0), w.double()
    l = xd @ wd.t()
    lp = torch.log_softmax(l, dim=1)
    h = torch.where(live, torch.special.entr(lp.exp()).sum(dim=1), 0.0)
    out = {"live": live, "lp": lp, "entropy": h, "x": xd}
    if tags is not None:
        out["logp"] = torch.where(tags >= 0, lp.gather(1, tags.clamp(min=0)), 0.0)
    if K:
        order = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :K]
        out["top"] = torch.where(live[:, None], order, -1)
        out["top_logp"] = torch.where(live[:, None], lp.gather(1, order), 0.0)
    return out


def d_of(want, tags, dlogp, dentropy):
    lp, live = want["lp"], want["live"]
    p = lp.exp()
    a = torch.where(tags >= 0, dlogp.double(), 0.0) if tags is not None else torch.zeros(p.shape[0], 1, dtype=torch.float64, device="cuda")
    b = torch.where(live, dentropy.double(), 0.0)[:, None] if dentropy is not None else 0.0
    d = -p * (a.sum(dim=1, keepdim=True) + b * (lp + want["entropy"][:, None]))
    d = torch.where(live[:, None], d, 0.0)
    return d.scatter_add_(1, tags.clamp(min=0), a) if tags is not None else d


def score_bound(x, w):
    """A score is off by at most its fp32 sum's error; the logarithm of the sum by as much, and by 2^-20 for the exponentials, the
    logarithm and the joining of tiles, all absolute.  Given and likeliest words' own scores have 64 bits, the largest score is taken
    off twice: once as the product gave it."""
    D = x.shape[1]
    worst = float((x.double().abs() @ w.double().abs().t()).nan_to_num(0, 0, 0).max()) if x.shape[0] else 0.0
    return 2 * 2.0 ** -24 * (math.sqrt(6 * D) + 4) * worst + 2.0 ** -20


def check_answers(x, w, tags, K, got, want=None):
    want = want or definition(x, w, tags, K)
    b = score_bound(want["x"], w)
    for k in ("logp", "top_logp"):
        if got[k] is not None:
            assert bool(((got[k].double() - want[k]).abs() <= b + 2.0 ** -23 * want[k].abs()).all()), k
    if K:
        assert torch.equal(got["top"], want["top"])
    if got["entropy"] is not None:
        # p (log p + H) over all words is at most 2 H, times the scores' error
        assert bool(((got["entropy"].double() - want["entropy"]).abs() <= (2 * want["entropy"] + 1) * b * want["live"]).all())
    return b


def check_gradients(x, w, tags, dlogp, dentropy, got, b, want, extra=0.0):
    d = d_of(want, tags, dlogp, dentropy)
    # a probability is off by the scores' error, log p + H by as much again; roundings to bf16: d and the result's own
    bound = ref.tol(x.dtype, max(x.shape[0], w.shape[0]), 2.25) + 4 * b + extra
    if got[0] is not None:
        ref.check("dx", got[0], d @ w.double(), bound)
    ref.check("dw", got[1], d.t() @ want["x"], bound)


def upstream(N, T, seed=5):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn((N, T), generator=gen) / N).cuda() if T else None, (0.1 * torch.randn(N, generator=gen) / N).cuda()


@dtypes
@pytest.mark.parametrize("N,D,V,T,K", SIZES)
def test_values_and_gradients(N, D, V, T, K, dtype):
    print(f"case logp {N} {D} {V} {T} {K} {dtype}", flush=True)
    x, w, tags = inputs(N, D, V, T, dtype)
    got = answers(x, w, tags, K)
    want = definition(x, w, tags, K)
    b = check_answers(x, w, tags, K, got, want)
    dlogp, dentropy = upstream(N, T)
    if T:
        dlogp[tags < 0] = float("nan")       # not looked at
        dentropy[~want["live"]] = float("nan")
        dlogp_ref = torch.where(tags >= 0, dlogp, 0.0)
        dent_ref = torch.where(want["live"], dentropy, 0.0)
    else:
        dlogp_ref, dent_ref = None, dentropy
    grads = gradients(x, w, tags, got, dlogp, dentropy)
    check_gradients(x, w, tags, dlogp_ref, dent_ref, grads, b, want)
    assert torch.equal(gradients(x, w, tags, got, dlogp, dentropy, want_dx=False)[1], grads[1])
    if T:
        only = gradients(x, w, tags, got, dlogp, None)
        check_gradients(x, w, tags, dlogp_ref, None, only, b, want)
        alone = answers(x, w, tags, 0, entropy=False, state=False)
        assert torch.equal(alone["logp"], got["logp"])


@dtypes
@pytest.mark.parametrize("N", [3, 90, 260])      # few rows, rows that stay where they are, rows that are gathered
def test_masked_rows_are_not_looked_at(N, dtype):
    x, w, tags = inputs(N, 70, 260, 2, dtype, seed=3, masked=0.5)
    tags[1] = -1
    off = (tags < 0).all(dim=1)
    dlogp, dentropy = upstream(N, 2)
    clean = answers(x, w, tags, 4)
    grads = gradients(x, w, tags, clean, dlogp, dentropy)
    x2 = x.clone()
    x2[off] = float("nan")
    x2[1] = float("inf")
    tags2 = torch.where(tags < 0, torch.full_like(tags, -(1 << 40)), tags)
    again = answers(x2, w, tags2, 4)
    for k in clean:
        assert torch.equal(clean[k], again[k]), k
    for a, b in zip(grads, gradients(x2, w, tags2, again, dlogp, dentropy)):
        assert torch.equal(a, b)
    assert not clean["entropy"][off].any() and not clean["logp"][off].any() and (clean["top"][off] == -1).all() and not grads[0][off].any()


@dtypes
@pytest.mark.parametrize("N", [1, 70, 193])
def test_no_row_left(N, dtype):
    x, w, tags = inputs(N, 33, 40, 2, dtype)
    tags.fill_(-1)
    x.fill_(float("nan"))
    got = answers(x, w, tags, 3)
    assert not got["logp"].any() and not got["entropy"].any() and (got["top"] == -1).all() and not got["top_logp"].any()
    dx, dw = gradients(x, w, tags, got, *upstream(N, 2))
    assert not dx.any() and not dw.any()


@dtypes
def test_no_rows(dtype):
    x, w, _ = inputs(0, 33, 40, 0, dtype)
    answers(x, w, None, 3)
    tags = torch.empty(0, 2, dtype=torch.int64, device="cuda")
    got = answers(x, w, tags, 3)
    dx, dw = gradients(x, w, tags, got, torch.empty(0, 2, device="cuda"), torch.empty(0, device="cuda"))
    assert not dw.any()


@dtypes
@pytest.mark.parametrize("N", [20, 50, 200])
def test_a_tag_outside_the_vocabulary_is_loud(N, dtype):
    x, w, tags = inputs(N, 40, 100, 2, dtype, masked=0.0)
    tags[7, 1], tags[8, 0] = 100, 1 << 40
    got = answers(x, w, tags, 3)
    assert torch.equal(torch.isnan(got["logp"]), tags >= 100) and not torch.isnan(got["entropy"]).any()
    dx, dw = gradients(x, w, tags, got, *upstream(N, 2))
    bad = (tags >= 100).any(dim=1)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all() and torch.isnan(dw).all()


@dtypes
@pytest.mark.parametrize("N", [8, 100])
@pytest.mark.parametrize("V", [40, 3001, 70001])
def test_equal_scores_come_in_the_vocabulary_s_order(N, V, dtype):
    """Whole numbers, so all scores are exact: rows of zeros (all words are alike), few different scores, words that repeat."""
    gen = torch.Generator().manual_seed(V)
    x = torch.randint(-2, 3, (N, 8), generator=gen).to(dtype)
    x[0] = 0
    x[1] = -1
    w = torch.randint(-2, 3, (V, 8), generator=gen).to(dtype)
    w[V // 2:V // 2 + 20] = w[3]
    if N > 6:
        w[:, 7] = 1.0
        x[5], x[6] = 0, 0
        x[5, 7], x[6, 7] = 3.0, -5.0       # all scores alike, above and below zero
    x, w = x.cuda(), w.cuda()
    for K in (1, 5, 33, min(V, 64)):
        got = answers(x, w, None, K)
        want = definition(x, w, None, K)
        assert torch.equal(got["top"], want["top"]), K
    # log p of exact scores: what the exponentials, their sum and its logarithm cost
    assert float((got["top_logp"].double() - want["top_logp"]).abs().max()) <= 2.0 ** -19
    assert float((got["entropy"].double() - want["entropy"]).abs().max()) <= 2.0 ** -19 * math.log(V) * 2


@dtypes
def test_near_scores_are_told_apart_in_64_bits(dtype):
    """Two hundred words within 2^-20 of each other, in an order that fp32 sums cannot see."""
    gen = torch.Generator().manual_seed(1)
    N, D, V = 40, 512, 5000
    w = torch.randn((V, D), generator=gen)
    near = torch.randperm(V, generator=gen)[:200]
    w[near] = w[near[0]].clone()
    w[near, torch.arange(200)] += 0.05 * (torch.arange(200) % 7 + 1)
    x = w[near[0]] * 0.3 + 0.05 * torch.randn((N, D), generator=gen)
    x[:, :200] = 1e-5 * torch.randn((N, 200), generator=gen)      # what tells them apart, 10^-6 of scores around 100
    x, w = x.to(dtype).cuda(), w.to(dtype).cuda()
    got = answers(x, w, None, 64)
    check_answers(x, w, None, 64, got)


@dtypes
def test_rows_that_are_sure_keep_their_digits(dtype):
    """One word with nearly all: log p and the entropy are as exact relative to themselves as the scores allow, down to 10^-20."""
    N, V = 40, 300
    x = torch.ones(N, 1)
    x[:, 0] = torch.linspace(1.0, 3.0, N)
    w = torch.full((V, 1), -16.0)
    w[::3] = -20.0
    w[77] = 0.0
    x, w = x.to(dtype).cuda(), w.to(dtype).cuda()
    tags = torch.full((N, 2), 77, device="cuda")
    tags[:, 1] = 5
    got = answers(x, w, tags, 2)
    l = x.double() @ w.double().t()
    others = torch.arange(V, device="cuda") != 77
    rest = torch.exp(l[:, others]).sum(dim=1)
    lp = -torch.log1p(rest)
    h = torch.log1p(rest) + (torch.exp(l[:, others]) * -l[:, others]).sum(dim=1) / (1 + rest)
    # one product a score: exact but for its rounding at up to 60, 2^-19; the exponential passes that on
    for a, b in ((got["logp"][:, 0], lp), (got["top_logp"][:, 0], lp), (got["entropy"], h)):
        assert float(((a.double() - b).abs() / b.abs()).max()) <= 2.0 ** -17
    dlogp, dentropy = torch.ones(N, 2, device="cuda"), None
    dlogp[:, 1] = 0.0
    want = definition(x, w, tags, 2)
    want["lp"] = want["lp"].clone()
    want["lp"][:, 77] = lp
    dx, dw = gradients(x, w, tags, got, dlogp, dentropy)
    d = -torch.exp(want["lp"])
    d[:, 77] = -torch.expm1(lp)
    bound = ref.tol(dtype, V, 2.25) + 2.0 ** -17
    ref.check("dw", dw, d.t() @ x.double(), bound)
    ref.check("dx", dx, d @ w.double(), bound)


@dtypes
@pytest.mark.parametrize("N", [6, 50])
def test_infinite_and_missing_numbers(N, dtype):
    """Words that no row can reach count for nothing; rows without a distribution are NaN, and only they."""
    x, w, _ = inputs(N, 33, 150, 0, dtype, seed=9, std=2.0)
    x[:, 0] = 1.0
    w[:, 0] = 0.0
    w[77] = 0.0
    w[77, 0] = float("-inf")
    tags = torch.randint(0, 150, (N, 2), generator=torch.Generator().manual_seed(2)).cuda()
    tags[tags == 77] = 3
    tags[2, 0] = 77
    x[4, 3] = float("nan")
    x[5, 0] = -1.0       # a score of +inf
    got = answers(x, w, tags, 64)
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[4] = bad[5] = True
    assert torch.isnan(got["logp"][bad]).all() and torch.isnan(got["entropy"][bad]).all() and (got["top"][bad] == -1).all() and torch.isnan(got["top_logp"][bad]).all()
    keep = torch.arange(150, device="cuda") != 77
    want = definition(x[~bad], w[keep], None, 64)
    top = got["top"][~bad]
    assert torch.equal(top - (top > 77).long(), want["top"])
    assert bool(((got["entropy"][~bad].double() - want["entropy"]).abs() <= (2 * want["entropy"] + 1) * score_bound(x[~bad], w[keep])).all())
    assert float(got["logp"][2, 0]) == float("-inf") and torch.isfinite(got["logp"][~bad]).sum() == 2 * int((~bad).sum()) - 1
    # all words out of reach
    w[:, 0] = float("-inf")
    got = answers(x, w, tags, 3)
    assert torch.isnan(got["entropy"]).all() and (got["top"] == -1).all()


@dtypes
def test_words_out_of_reach_may_be_asked_for(dtype):
    """Fewer words with a score than are asked for: the others follow, with log p = -inf, in their order."""
    x = torch.ones(3, 1).to(dtype).cuda()
    w = torch.full((100, 1), float("-inf")).to(dtype).cuda()
    w[60], w[20] = 2.0, 1.0
    got = answers(x, w, None, 5)
    assert got["top"].tolist() == [[60, 20, 0, 1, 2]] * 3
    assert torch.isinf(got["top_logp"][:, 2:]).all() and torch.isfinite(got["top_logp"][:, :2]).all()


def test_gradients_against_differences():
    N, T = 40, 3
    x, w, tags = inputs(N, 60, 90, T, torch.float32, seed=10)
    dlogp, dentropy = upstream(N, T)
    got = answers(x, w, tags, 0)
    dx, dw = gradients(x, w, tags, got, dlogp, dentropy)
    gen = torch.Generator().manual_seed(5)
    ex, ew = (torch.randn(a.shape, generator=gen, dtype=torch.float64).cuda() for a in (x, w))
    live = (tags >= 0).any(dim=1)

    def cost(e):
        want = definition(x.double() + e * ex, w.double() + e * ew, tags, 0)
        return float((want["logp"] * dlogp).sum() + (want["entropy"] * dentropy * live).sum())

    quotient = (cost(1e-5) - cost(-1e-5)) / 2e-5
    inner = float((dx.double() * ex).sum() + (dw.double() * ew).sum())
    size = float(dx.double().norm() * ex.norm() + dw.double().norm() * ew.norm())
    assert abs(inner - quotient) <= (ref.tol(torch.float32, 90, 0) + 4 * score_bound(x, w)) * size


def test_one_given_word_has_the_gradients_of_the_cross_entropy():
    """dlogp = -1 / N: what xent_fwd_bwd gives."""
    x, w, tags = inputs(70, 64, 500, 1, torch.float32, seed=4, masked=0.0)
    tags.clamp_(min=0)
    got = answers(x, w, tags, 0)
    dx, dw = gradients(x, w, tags, got, torch.full((70, 1), -1.0 / 70, device="cuda"), None)
    loss, cost, ex, ew = blank((70,)), blank((1,)), blank(x.shape), blank(w.shape)
    ws = torch.empty(lc.xent_workspace_bytes(70, 64, 500, lc.LC_F32, True), dtype=torch.uint8, device="cuda")
    lc.xent_fwd_bwd(x, w, tags[:, 0].contiguous(), None, loss, cost, ex, ew, lc.LC_F32, ws)
    b = score_bound(x, w)
    assert float((loss + got["logp"][:, 0]).abs().max()) <= 2 * b
    ref.check("dx", dx, ex, 2 * (ref.tol(torch.float32, 500, 0) + 2 * b))
    ref.check("dw", dw, ew, 2 * (ref.tol(torch.float32, 500, 0) + 2 * b))


@pytest.mark.parametrize("dtype,N,V", [(torch.bfloat16, 6000, 200001), (torch.float32, 3100, 200001)], ids=["bf16", "f32"])
def test_more_rows_than_are_kept_at_a_time(dtype, N, V):
    """d of all rows exceeds what is kept at once: the weight gradient adds up over blocks of rows; and rows in several blocks forward."""
    D, T, K = 72, 2, 3
    print(f"case logp blocks {N} {D} {V} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((N, D), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((V, D), generator=gen, device="cuda") * 2 * D ** -0.5).to(dtype)
    tags = torch.randint(0, V, (N, T), generator=gen, device="cuda")
    tags[torch.rand(N, generator=gen, device="cuda") < 0.1] = -1
    dlogp, dentropy = upstream(N, T)
    got = answers(x, w, tags, K)
    dx, dw = gradients(x, w, tags, got, dlogp, dentropy)
    rw, b = torch.zeros(V, D, device="cuda", dtype=torch.float64), score_bound(x[:500], w) * 1.2
    bound = ref.tol(dtype, V, 2.25) + 4 * b
    for i in range(0, N, 1000):
        at = slice(i, i + 1000)
        want = definition(x[at], w, tags[at], K)
        assert torch.equal(got["top"][at], want["top"])
        assert float((got["logp"][at].double() - want["logp"]).abs().max()) <= b + 2.0 ** -18
        d = d_of(want, tags[at], dlogp[at], dentropy[at])
        ref.check("dx", dx[at], d @ w.double(), bound)
        rw += d.t() @ want["x"]
    ref.check("dw", dw, rw, bound)


def test_rows_in_blocks_forward():
    """The groups' scores of all rows exceed what is kept at once."""
    N, V = 600, 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(1)
    N = 2500
    x = torch.randn((N, 8), generator=gen, device="cuda").to(torch.bfloat16)
    w = torch.randn((V, 8), generator=gen, device="cuda").to(torch.bfloat16)
    got = answers(x, w, None, 3)
    for i in (0, 2040, 2048, N - 20):
        want = definition(x[i:i + 20], w, None, 3)
        assert torch.equal(got["top"][i:i + 20], want["top"])


@dtypes
@pytest.mark.parametrize("N", [7, 130])
def test_the_same_bits_on_another_stream_and_in_a_graph(N, dtype):
    D, V, T, K = 100, 700, 2, 5
    x, w, tags = inputs(N, D, V, T, dtype, seed=11)
    dlogp, dentropy = upstream(N, T)
    first = answers(x, w, tags, K)
    first["dx"], first["dw"] = gradients(x, w, tags, first, dlogp, dentropy)
    out = {k: torch.empty_like(v) for k, v in first.items()}
    ws = torch.empty(lc.logp_workspace_bytes(N, D, V, T, K, code(dtype), True), dtype=torch.uint8, device="cuda")

    def both():
        lc.logp_fwd(x, w, tags, out["logp"], out["entropy"], out["top"], out["top_logp"], out["state"], code(dtype), ws)
        lc.logp_bwd(x, w, tags, out["logp"], out["state"], dlogp, dentropy, out["dx"], out["dw"], code(dtype), ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    for k in first:
        assert torch.equal(first[k], out[k]), k
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        ws.fill_(255)
        for v in out.values():
            v.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for k in first:
            assert torch.equal(first[k], out[k]), k


@dtypes
def test_tags_may_start_at_any_row_of_a_list(dtype):
    x, w, tags = inputs(21, 40, 100, 1, dtype, masked=0.2)
    longer = torch.full((24, 1), -9, dtype=torch.int64, device="cuda")
    longer[1:22] = tags
    a, b = answers(x, w, tags, 2), answers(x, w, longer[1:22], 2)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_more_rows_than_are_counted_at_a_time():
    """Rows with and without words, well beyond 8192, in an order that has no pattern."""
    N, D, V = 20000, 16, 40
    x, w, tags = inputs(N, D, V, 2, torch.float32, seed=21, masked=0.4)
    got = answers(x, w, tags, 2)
    check_answers(x, w, tags, 2, got)
    dlogp, dentropy = upstream(N, 2)
    want = definition(x, w, tags, 2)
    check_gradients(x, w, tags, dlogp, dentropy, gradients(x, w, tags, got, dlogp, dentropy), score_bound(want["x"], w), want)
