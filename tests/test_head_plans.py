"""Launch plans of the supervised head, checked on the host (no GPU): head_plan_query runs an operator's planning with every host
check, and the scratch that the planned kernels use is counted here apart from the sources."""
import math
import random

import pytest

import paper_1502_03409_amd as lc
from paper_1502_03409_amd import binding as B

TYPES = [lc.LC_F32, lc.LC_BF16]


def up(a, b):
    return -(-a // b) * b


def parts_bytes(plans):
    """What the sums of a cut product's parts take: [parts][rows][columns, to a multiple of 4] floats, one product at a time.  A product of
    tiles has its tile among its compile-time parameters and rows, columns, contraction and parts among its scalars."""
    cut = [p["arg"] for p in plans if p["tparam"][3] in (128, 256) and p["arg"][3] > 1]
    return max([4 * parts * rows * up(columns, 4) for rows, columns, _, parts, *_ in cut], default=0)


def xent_bytes(plans, N, D, V, dtype):
    """Least scratch of a loss with gradients: the rows that count, the weights unless used where they are, statistics and d of a block,
    parts, and the fp32 gradient that blocks are added up in."""
    es, planes = (2, 1) if dtype == lc.LC_BF16 else (4, 3)
    blocks = [p["arg"][0] for p in plans if p["kernel"] in ("xent", "xent (few rows)")]
    assert sum(blocks) == N
    block, Dp, Vp = max(blocks), up(D, 8), up(V, 64)
    used = 2 * planes * (N * Dp + block * Vp) + 8 * block * -(-V // 128) + parts_bytes(plans)
    if planes == 3:
        used += 4 * block * Vp
    if planes == 3 or D != Dp:
        used += 2 * planes * V * Dp
    return used + (4 * V * D if len(blocks) > 1 else 0)


def blocks_of(V, dtype):
    """Rows of a block of 2 GiB, in steps of 256."""
    return max(64, (2 << 30) // (up(V, 64) * (2 if dtype == lc.LC_BF16 else 4)) // 256 * 256)


# one block and several, the last one full, of one row, and in between
ROWS = [lambda b: 3 * b, lambda b: b + 1, lambda b: b + 33, lambda b: b + b // 10, lambda b: b + b // 2, lambda b: 2 * b - 7]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("D,V", [(66, 247098), (66, 80377), (475, 144808), (4096, 128000), (1024, 200000), (768, 300001)])
def test_blocks_of_rows_have_room_for_the_parts_of_each(D, V, dtype):
    for rows in ROWS:
        N = rows(blocks_of(V, dtype))
        plans = lc.head_plan_query(B.LC_HEAD_XENT_FWD_BWD, N, D, V, dtype)
        assert xent_bytes(plans, N, D, V, dtype) <= lc.xent_workspace_bytes(N, D, V, dtype, True), N


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_any_size_passes_the_host_checks_and_fits_its_scratch(dtype):
    rng = random.Random(5)
    for _ in range(1500):
        N, D, V = log_int(rng, 1, 30000), log_int(rng, 1, 16384), log_int(rng, 1, 300000)
        plans = lc.head_plan_query(B.LC_HEAD_XENT_FWD_BWD, N, D, V, dtype)
        assert xent_bytes(plans, N, D, V, dtype) <= lc.xent_workspace_bytes(N, D, V, dtype, True), (N, D, V)
        lc.head_plan_query(B.LC_HEAD_XENT_FWD, N, D, V, dtype)
        F = log_int(rng, 1, 16384)
        lc.head_plan_query(B.LC_HEAD_GLU_FWD, N, D, F, dtype)
        planes, es = (1, 2) if dtype == lc.LC_BF16 else (3, 4)
        used = parts_bytes(lc.head_plan_query(B.LC_HEAD_GLU_BWD, N, D, F, dtype)) + 2 * planes * N * 2 * up(F, 64)
        assert used <= lc.glu_workspace_bytes(N, D, F, dtype, True), (N, D, F)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_scratch_for_a_batch_is_enough_for_smaller_ones(dtype):
    """The last batch of an epoch, through the scratch of the others; fewer rows are cut into more parts."""
    rng = random.Random(6)
    sizes = [(1024, 2048, 192), (2048, 20011, 192), (400, 256, 512), (256, 1000, 512), (1024, 4096, 1024), (4096, 20011, 1024),
             (4096, 8192, 512), (8192, 20011, 512)]
    sizes += [(log_int(rng, 1, 8192), log_int(rng, 1, 200000), log_int(rng, 2, 8192)) for _ in range(150)]
    for D, width, N in sizes:
        for size in (lc.glu_workspace_bytes, lc.xent_workspace_bytes):
            for grads in (False, True):
                enough = size(N, D, width, dtype, grads)
                fewer = range(0, N) if N <= 1024 else [rng.randrange(N) for _ in range(200)] + list(range(N - 300, N))
                assert all(size(n, D, width, dtype, grads) <= enough for n in fewer), (size.__name__, D, width, N, grads)
            assert size(N, D, width, dtype, False) <= size(N, D, width, dtype, True)


def test_few_rows_ask_for_no_copy_of_the_weights():
    """Answers for up to 32 rows read the weights where they are; what is left are a few numbers for each row, and for each row and 64 words."""
    for dtype in TYPES:
        for N in (1, 5, 32):
            for D in (4096, 4097, 100):
                assert lc.glu_workspace_bytes(N, D, 8192, dtype) <= 4096
                assert lc.xent_workspace_bytes(N, D, 100003, dtype) <= 8 * up(N, 8) * (100003 // 64 + 1) + 16384
        assert lc.xent_workspace_bytes(33, 4097, 100003, dtype) > 100003 * 4097 * 2      # laid out from 33 rows on


def test_refusals():
    for op, sizes, dtype in ((9, (4, 4, 4), 0), (0, (-1, 4, 4), 0), (2, (4, 0, 4), 0), (3, (4, 4, 1 << 21), 1), (1, (4, 4, 4), 5)):
        with pytest.raises(lc.LcError) as e:
            lc.head_plan_query(op, *sizes, dtype)
        assert e.value.code == B.LC_EINVAL
