"""Rows, weights and stacks of the head's largest sizes, planned on the host: they are laid out by launches of fewer than 2^32 threads, and scratch
is no more than is said."""
import math
import random

import pytest

import paper_1502_03409_amd as lc
from paper_1502_03409_amd import binding as B

TYPES = [lc.LC_F32, lc.LC_BF16]


def laid_out(plans, kernel):
    """Threads of the launches of `kernel`, which take 8 values each; every launch of the plan is one that the runtime accepts."""
    for p in plans:
        assert p["grid"][0] * p["block"] < 1 << 32, p
    return sum(p["grid"][0] * p["block"] for p in plans if p["kernel"] == kernel)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("op,kernel", [(B.LC_HEAD_LOGP_FWD, "logp (w)"), (B.LC_HEAD_LOGP_BWD, "logp (w)"), (B.LC_HEAD_XENT_FWD, "xent (w)"),
                                       (B.LC_HEAD_XENT_FWD_BWD, "xent (w)")])
def test_weights(op, kernel, dtype):
    """Widths that are no multiple of eight are laid out in either type."""
    for V, D in ((1 << 20, (1 << 15) - 1), (1 << 20, (1 << 15) + 5), (1 << 20, 1 << 17), ((1 << 20) - 3, (1 << 14) - 1)):
        if D % 8 or dtype == lc.LC_F32:
            threads = laid_out(lc.head_plan_query(op, 64, D, V, dtype), kernel)
            assert 0 <= threads - V * (-(-D // 8)) < 256, (V, D)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_rows_weights_and_gradients_of_the_gated_layer(dtype):
    for N, D, F in ((1 << 24, 2047, 64), ((1 << 24) - 5, 1023, 64), (1 << 24, 65, 1000)):
        plans = lc.head_plan_query(B.LC_HEAD_GLU_BWD, N, D, F, dtype)
        assert 0 <= laid_out(plans, "glu (x, w)") - (N + 2 * F) * (-(-D // 8)) < 256
        assert 0 <= laid_out(plans, "glu_bwd (gradients)") - N * (-(-F // 64) * 8) < 256


# 2^32 and 2^33 threads; just below, at and behind what one launch takes
SIZES = [(1 << 24, 2048), (1 << 24, 4096), (1 << 24, 1024), ((1 << 24) - 1, 1024), ((1 << 24) - 77, 1032)]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D", SIZES)
def test_gathered_rows_of_the_answers(N, D, dtype):
    for op in (B.LC_HEAD_LOGP_FWD, B.LC_HEAD_LOGP_BWD):
        threads = laid_out(lc.head_plan_query(op, N, D, 5, dtype), "logp_gather")
        assert 0 <= threads - N * (D // 8) < 256


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D", SIZES)
def test_gathered_rows_of_the_loss(N, D, dtype):
    for op in (B.LC_HEAD_XENT_FWD, B.LC_HEAD_XENT_FWD_BWD):
        threads = laid_out(lc.head_plan_query(op, N, D, 5, dtype), "xent_gather")
        assert 0 <= threads - N * (D // 8) < 256


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_scratch_of_a_stack_is_bounded(dtype):
    """4 GiB, or what one matrix takes; sides that differ little have the most places of the short side's square beside X's."""
    rng = random.Random(10)
    shapes = [(5000, 1000, 1001), (100000, 130, 131), (65536, 600, 601), (1 << 20, 128, 128), (1 << 24, 1, 1), (1 << 24, 3, 300), (40, 5000, 4500)]
    for _ in range(400):
        rows, cols = (int(round(math.exp(rng.uniform(0, math.log(30000))))) for _ in range(2))
        shapes.append((rng.randrange(1, 1 << 24), rows, rng.choice([cols, rows, rows + 1])))
    for count, rows, cols in shapes:
        count = min(count, (1 << 40) // (rows * cols))
        one, all_of_them = (lc.muon_workspace_bytes(n, rows, cols, dtype) for n in (1, count))
        assert 0 < all_of_them <= max(one, 4 << 30), (count, rows, cols, all_of_them / 2 ** 30)
