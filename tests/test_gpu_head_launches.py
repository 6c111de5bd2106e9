"""Rows that are laid out by more than one launch: a launch takes 2^31 threads of eight values each.  Rows on both sides of what the first one
takes, and the last ones, against the definitions in 64 bits."""
import pytest
import torch

import head_ref as ref
import test_gpu_glu as G
import test_gpu_logp as logp
import test_gpu_xent as X

pytestmark = pytest.mark.gpu


def rows_to_look_at(N, pieces):
    border = (1 << 31) // pieces
    assert 100 < border < N - 300
    return torch.cat([torch.arange(a, b, device="cuda") for a, b in ((0, 100), (border - 100, border + 100), (N - 100, N))])


def normal(shape, std, seed):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, std, generator=torch.Generator("cuda").manual_seed(seed))


def test_rows_of_the_gated_layer():
    N, D, F = 1 << 23, 2051, 24
    print(f"case glu {N} x {D} -> {F}", flush=True)
    x, wg, wu = normal((N, D), 1.0, 0), normal((F, D), D ** -0.5, 1), normal((F, D), D ** -0.5, 2)
    h, _ = G.forward(x, wg, wu, "silu", save=False)
    at = rows_to_look_at(N, 257)
    ref.check("h", h[at], ref.glu(x[at], wg, wu, "silu")[0], ref.tol(torch.bfloat16, D, 1))


def test_rows_of_the_answers_and_their_gradients():
    N, D, V = 1 << 24, 1030, 5
    print(f"case logp {N} x {D} over {V} words", flush=True)
    x, w = normal((N, D), 1.0, 3), normal((V, D), 2 * D ** -0.5, 4)
    tags = torch.arange(N, device="cuda")[:, None] % (V + 1) - 1
    at = rows_to_look_at(N, 129)
    got = logp.answers(x, w, tags, 2)
    few = {k: v[at] for k, v in got.items()}
    want = logp.definition(x[at], w, tags[at], 2)
    b = logp.check_answers(x[at], w, tags[at], 2, few, want)
    dlogp, dentropy = normal((N, 1), 1.0, 5).float(), normal((N,), 1.0, 6).float()
    dx, _ = logp.gradients(x, w, tags, got, dlogp, dentropy)
    assert not dx[at][~want["live"]].any()
    d = logp.d_of(want, tags[at], dlogp[at], dentropy[at])
    ref.check("dx", dx[at], d @ w.double(), ref.tol(torch.bfloat16, V, 2.25) + 4 * b)   # roundings and scores as in the tests of small sizes


def test_rows_of_the_loss():
    N, D, V = 1 << 24, 1030, 5
    print(f"case xent {N} x {D} over {V} words", flush=True)
    x, w = normal((N, D), 1.0, 7), normal((V, D), 2 * D ** -0.5, 8)
    target, scale = torch.arange(N, device="cuda") % (V + 1) - 1, torch.ones(N, device="cuda")
    at = rows_to_look_at(N, 129)
    loss, _, dx, _ = X.run(x, w, target, scale)
    want, _, want_dx, _ = ref.xent(x[at], w, target[at], scale[at])
    b = X.loss_bound(x[at], w)
    assert float((loss[at].double() - want).abs().max()) <= b + 2.0 ** -23 * float(want.max())
    assert not dx[at][target[at] < 0].any()
    ref.check("dx", dx[at], want_dx, ref.tol(torch.bfloat16, V, 2.25) + b)   # as at small sizes
