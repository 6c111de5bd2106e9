"""Rows that are laid out by more than one launch: a launch takes 2^31 threads of eight values each.  Rows on both sides of what the first one
takes, and the last ones, against the definitions in 64 bits."""
import pytest
import torch

import head_ref as ref
import test_gpu_glu as G

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
