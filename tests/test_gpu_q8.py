"""q8_rows, q8_matmul and q8_glu_fwd against their definitions in 64 bits."""
import pytest
import torch

import head_ref as ref
import paper_1502_03409_amd as lc

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
ACTS = {"sigmoid": lc.LC_ACT_SIGMOID, "silu": lc.LC_ACT_SILU, "gelu": lc.LC_ACT_GELU}
# one row to tiles of 128 and 256, widths around blocks of 16, 32, 128 and one
SIZES = [(1, 1, 1), (1, 128, 64), (2, 129, 33), (8, 127, 31), (9, 640, 65), (32, 1000, 260), (33, 200, 129), (64, 128, 1000), (130, 333, 257),
         (300, 520, 515)]


def code(dtype):
    return lc.LC_BF16 if dtype == torch.bfloat16 else lc.LC_F32


def ids(dtype):
    return "bf16" if dtype == torch.bfloat16 else "f32"


def q8(x):
    """Whole numbers and scales of rows, in 64 bits but for the scale's one rounding to 32.  Tensors divide tensors: torch divides by a number
    with a product by its rounded reciprocal."""
    amax = x.float().abs().amax(dim=1)
    s = (amax.double() / torch.full_like(amax, 127, dtype=torch.float64)).float().clamp(min=2.0 ** -126)
    q = torch.round(x.double() / s.double()[:, None]).clamp(-127, 127)
    bad = ~torch.isfinite(amax)
    return torch.where(bad[:, None], 0.0, q), torch.where(bad, float("nan"), s)


def rows(x):
    q = torch.full((x.shape[0], lc.q8_row_bytes(x.shape[1])), 99, dtype=torch.int8, device="cuda")
    s = torch.full((x.shape[0],), -1.0, device="cuda")
    lc.q8_rows(x, q, s, code(x.dtype))
    return q, s


def scratch(N, D, F, dtype):
    return torch.full((lc.q8_workspace_bytes(N, D, F, code(dtype)),), 0x7b, dtype=torch.uint8, device="cuda")


def draw(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def matmul(x, q, s):
    y = torch.full((x.shape[0], q.shape[0]), float("nan"), dtype=x.dtype, device="cuda")
    lc.q8_matmul(x, q, s, y, code(x.dtype), scratch(x.shape[0], x.shape[1], q.shape[0], x.dtype))
    return y


def glu(x, qg, sg, qu, su, act):
    h = torch.full((x.shape[0], qg.shape[0]), float("nan"), dtype=x.dtype, device="cuda")
    lc.q8_glu_fwd(x, qg, sg, qu, su, h, ACTS[act], code(x.dtype), scratch(x.shape[0], x.shape[1], qg.shape[0], x.dtype))
    return h


def want_matmul(x, w):
    qx, sx = q8(x)
    qw, sw = q8(w)
    return (qx @ qw.t()) * sx.double()[:, None] * sw.double()[None, :]


def close(got, want):
    """Every value: the exact sum, rounded to fp32, times two scales, each product rounded, then rounded to the result's type; and what
    the smallest normal numbers lose."""
    step = 3 * 2.0 ** -24 + (2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0)
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = torch.isfinite(want)
    assert ((got - want).abs()[fine] <= want.abs()[fine] * step * (1 + 2.0 ** -6) + 2.0 ** -133).all()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("N,D", [(1, 1), (1, 127), (3, 128), (5, 129), (70, 1000), (2, 9001), (300, 72)])
def test_rows(N, D, dtype):
    print(f"case q8_rows {N} {D} {dtype}", flush=True)
    x = draw((N, D), dtype, N + D)
    x[0, D // 2] = 0.0
    q, s = rows(x)
    wq, ws = q8(x)
    assert torch.equal(s, ws) and torch.equal(q[:, :D].double(), wq) and not q[:, D:].any()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_rows_on_and_next_to_halves(dtype):
    """Scales that are and are not powers of two, values on every half and its neighbours on both sides."""
    k = torch.arange(-127, 127, dtype=torch.float64) + 0.5
    x = []
    for top in (127.0, 254.0, 100.0, 1.0, 3e-30, 1e30):
        s = float((torch.tensor(top).to(dtype).float() / 127).double())
        at = (k * s).to(dtype)
        for v in (at, torch.nextafter(at.float(), torch.tensor(float("inf"))).to(dtype), torch.nextafter(at.float(), torch.tensor(-float("inf"))).to(dtype)):
            row = torch.cat([torch.tensor([top]).to(dtype), v.clamp(-top, top)])
            x.append(row)
    x = torch.stack(x).cuda()
    q, s = rows(x)
    wq, ws = q8(x)
    assert torch.equal(s, ws) and torch.equal(q[:, :x.shape[1]].double(), wq)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_rows_of_zeros_tiny_values_and_no_numbers(dtype):
    x = torch.zeros(6, 40, dtype=dtype)
    x[1, 3] = 1e-40
    x[2, 39] = float("inf")
    x[3, 0] = float("nan")
    x[4, 7] = torch.finfo(dtype).max
    x[5] = 2.0 ** -120
    x = x.cuda()
    q, s = rows(x)
    wq, ws = q8(x)
    assert torch.equal(torch.nan_to_num(s, -1.0), torch.nan_to_num(ws, -1.0)) and torch.equal(q[:, :40].double(), wq)
    w = draw((70, 40), dtype, 1)
    qw, sw = rows(w)
    sw[5] = float("nan")
    y = matmul(x, qw, sw)
    assert torch.isnan(y[2:4]).all() and torch.isnan(y[:, 5]).all() and not torch.isnan(y[4:, 6:]).any() and not y[0, 6:].any()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("N,D,F", SIZES)
def test_matmul(N, D, F, dtype):
    print(f"case q8_matmul {N} {D} {F} {dtype}", flush=True)
    x, w = draw((N, D), dtype, 3), draw((F, D), torch.float32, 4, D ** -0.5)
    q, s = rows(w)
    close(matmul(x, q, s), want_matmul(x, w))


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("N,D,F", [(1, 1, 1), (5, 100, 17), (32, 256, 64), (33, 130, 31), (140, 300, 290), (300, 128, 515)])
def test_gated_layer(N, D, F, act, dtype):
    print(f"case q8_glu {N} {D} {F} {act} {dtype}", flush=True)
    x, wg, wu = draw((N, D), dtype, 5), draw((F, D), torch.float32, 6, 2 * D ** -0.5), draw((F, D), torch.float32, 7, D ** -0.5)
    (qg, sg), (qu, su) = rows(wg), rows(wu)
    g, u = want_matmul(x, wg), want_matmul(x, wu)
    # g and u are off by 3 2^-24 of themselves; a gate of |g| < 2^4 passes that on at most 16-fold, its own forms cost a few more
    bound = 64 * 2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    ref.check("h", glu(x, qg, sg, qu, su, act), ref.act(act, g)[0] * u, bound)


def test_largest_sums():
    """2^17 products of 127 x 127 stay whole numbers of 31 bits."""
    D = 1 << 17
    x, w = torch.ones(33, D, device="cuda"), torch.full((40, D), -1.0, device="cuda")
    q, s = rows(w)
    y = matmul(x, q, s)
    close(y, want_matmul(x, w))
    close(matmul(x[:3].contiguous(), q, s), want_matmul(x[:3], w))
    with pytest.raises(lc.LcError):
        lc.q8_matmul(torch.zeros(1, D + 1, device="cuda"), torch.zeros(1, 0, dtype=torch.int8, device="cuda"), s[:1], y[:1, :1].contiguous(), lc.LC_F32, s)


@pytest.mark.parametrize("N", [7, 200])
def test_what_lies_around_is_left_alone_and_calls_repeat(N):
    x, w = draw((N, 200), torch.bfloat16, 1), draw((301, 200), torch.float32, 2)
    q, s = rows(w)
    room = torch.full((N + 2, 301), 7.0, dtype=torch.bfloat16, device="cuda")
    flat = room.view(-1)[304:304 + N * 301].view(N, 301)
    ws = scratch(N, 200, 301, torch.bfloat16)
    lc.q8_matmul(x, q, s, flat, lc.LC_BF16, ws)
    assert (room.view(-1)[:304] == 7).all() and (room.view(-1)[304 + N * 301:] == 7).all()
    close(flat, want_matmul(x, w))
    first = flat.clone()
    ws.fill_(0)
    lc.q8_matmul(x, q, s, flat, lc.LC_BF16, ws)
    assert torch.equal(first, flat)
    # q's own bytes behind a row need not be looked after by x: its are zeros
    q[:, 200:] = 55
    lc.q8_matmul(x, q, s, flat, lc.LC_BF16, ws)
    assert torch.equal(first, flat)


def test_no_rows():
    q, s = rows(draw((5, 9), torch.float32, 0))
    assert matmul(torch.empty(0, 9, device="cuda"), q, s).shape == (0, 5)
    assert glu(torch.empty(0, 9, device="cuda"), q, s, q, s, "silu").shape == (0, 5)


@pytest.mark.parametrize("N", [3, 150])
def test_captured_and_replayed(N):
    x, w = draw((N, 140), torch.bfloat16, 8), draw((270, 140), torch.float32, 9)
    q, s = rows(w)
    y, h = (torch.empty(N, 270, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = scratch(N, 140, 270, torch.bfloat16)

    def both():
        lc.q8_matmul(x, q, s, y, lc.LC_BF16, ws)
        lc.q8_glu_fwd(x, q, s, q, s, h, lc.LC_ACT_SILU, lc.LC_BF16, ws)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (10, 11, 12):
        x.copy_(draw((N, 140), torch.bfloat16, seed))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), h.clone()
        both()
        torch.cuda.synchronize()
        assert torch.equal(got[0], y) and torch.equal(got[1], h)
