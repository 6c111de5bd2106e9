"""The head's operators where its products take large tiles, or are cut along a long contraction: sizes that no tile divides, against
64 bits on the GPU.  The operators' other tests are at sizes of small tiles."""
import pytest
import torch

import head_ref as ref
import paper_1502_03409_amd as lc
import test_gpu_glu as G
import test_gpu_xent as X

pytestmark = pytest.mark.gpu

# rows, features, hidden: wide results of the forward product, of dx, of the weight gradients, and long contractions over few tiles
GLU = [(8203, 72, 4105), (8203, 8200, 41), (75, 8203, 4101), (90, 200, 9000), (9001, 130, 70)]
# rows, features, words: wide scores, wide dx, wide dw, long contractions of dx and of dw
XENT = [(8203, 72, 8301), (8203, 8201, 99), (93, 8200, 8203), (41, 130, 30011), (9001, 70, 130)]


@G.dtypes
@pytest.mark.parametrize("N,D,F", GLU)
def test_glu(N, D, F, dtype):
    print(f"case large glu {N} {D} {F} {dtype}", flush=True)
    x, wg, wu, dh = G.inputs(N, D, F, dtype, seed=1)
    h, gu = G.forward(x, wg, wu, "silu")
    ref.check("h", h, ref.glu(x, wg, wu, "silu")[0], ref.tol(dtype, D, 1))
    dx, dwg, dwu = G.backward(x, wg, wu, gu, dh, "silu")
    rx, rwg, rwu = ref.glu_grads(x, wg, wu, dh, "silu")
    # roundings as at small sizes
    ref.check("dx", dx, rx, ref.tol(dtype, D + 2 * F, 2.75))
    ref.check("dwg", dwg, rwg, ref.tol(dtype, D + N, 2.75))
    ref.check("dwu", dwu, rwu, ref.tol(dtype, D + N, 2.75))


@X.dtypes
@pytest.mark.parametrize("masked", [0.1, 0.995], ids=["most_rows", "few_rows"])
@pytest.mark.parametrize("N,D,V", XENT)
def test_xent(N, D, V, masked, dtype):
    print(f"case large xent {N} {D} {V} {masked} {dtype}", flush=True)
    x, w, t = X.inputs(N, D, V, dtype, seed=2, masked=masked)
    t[N // 2] = V - 1
    got = X.run(x, w, t)
    X.check_all(x, w, t, None, got)
    loss, cost = X.run(x, w, t, grads=False)
    assert torch.equal(loss, got[0]) and torch.equal(cost, got[1])


def test_infinities_in_large_tiles_of_fp32():
    """A row with an infinity is formed again with the fp32 instruction; its neighbours in the tile stay what they are."""
    N, D, F = 8203, 72, 4105
    x, wg, wu, _ = G.inputs(N, D, F, torch.float32, seed=3)
    clean, _ = G.forward(x, wg, wu, "sigmoid", save=False)
    x[5000, 3], x[8202, 71], x[17, 0] = float("inf"), float("-inf"), float("nan")
    h, gu = G.forward(x, wg, wu, "sigmoid")
    rh, rg, ru = ref.glu(x, wg, wu, "sigmoid")
    ref.check("g", gu[:, 0], rg, ref.tol(torch.float32, D, 0))
    ref.check("u", gu[:, 1], ru, ref.tol(torch.float32, D, 0))
    keep = torch.ones(N, dtype=torch.bool, device="cuda")
    keep[[5000, 8202, 17]] = False
    ref.check("other rows", h[keep], rh[keep], ref.tol(torch.float32, D, 1))


def test_infinite_weights_in_gradients_of_fp32():
    """Contractions over rows of a matrix (products by columns) with an infinity among them."""
    x, wg, wu, dh = G.inputs(40, 96, 200, torch.float32, seed=4)
    _, gu = G.forward(x, wg, wu, "silu")
    x2, wg2 = x.clone(), wg.clone()
    x2[7, 11] = float("inf")
    wg2[3, 5] = float("-inf")
    dx, dwg, dwu = G.backward(x2, wg2, wu, gu, dh, "silu")
    a, da = ref.act("silu", gu[:, 0].double())
    dg, du = dh.double() * gu[:, 1].double() * da, dh.double() * a
    ref.check("dx", dx, dg @ wg2.double() + du @ wu.double(), ref.tol(torch.float32, 500, 0))
    ref.check("dwg", dwg, dg.t() @ x2.double(), ref.tol(torch.float32, 140, 0))
    ref.check("dwu", dwu, du.t() @ x2.double(), ref.tol(torch.float32, 140, 0))


@G.dtypes
@pytest.mark.parametrize("N,D,F", [(150, 61952, 70), (20, 93312, 40)])
def test_features_of_whole_layers(N, D, F, dtype):
    """As many features as the pooled responses of a layer have, e.g. 44 x 44 places of 32 filters: one long contraction forward, wide
    gradients."""
    print(f"case wide glu {N} {D} {F} {dtype}", flush=True)
    x, wg, wu, dh = G.inputs(N, D, F, dtype, seed=5)
    h, gu = G.forward(x, wg, wu, "silu")
    ref.check("h", h, ref.glu(x, wg, wu, "silu")[0], ref.tol(dtype, D, 1))
    dx, dwg, dwu = G.backward(x, wg, wu, gu, dh, "silu")
    rx, rwg, rwu = ref.glu_grads(x, wg, wu, dh, "silu")
    ref.check("dx", dx, rx, ref.tol(dtype, D + 2 * F, 2.75))
    ref.check("dwg", dwg, rwg, ref.tol(dtype, D + N, 2.75))
    ref.check("dwu", dwu, rwu, ref.tol(dtype, D + N, 2.75))
