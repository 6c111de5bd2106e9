"""Answers of the softmax, orthogonalised steps and 8-bit weights on the host: arguments are refused before anything is launched,
workspaces hold what the planned kernels use, and all plans pass their checks."""
import math
import random

import pytest
import torch

import paper_1502_03409_amd as lc
from paper_1502_03409_amd import binding as B
from paper_1502_03409_amd import head as H

P = 0x10000      # an aligned address that is never used: every call below is refused, or has nothing to do
BIG = 1 << 50    # a workspace size that is always enough
TYPES = [lc.LC_F32, lc.LC_BF16]


def L():
    return H._lib()


def caller(fn, ok):
    def call(i=None, v=None):
        a = list(ok)
        if i is not None:
            a[i] = v
        return fn(*a)
    return call


def up(a, b):
    return -(-a // b) * b


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# x w tags logp entropy top top_logp state | N D V T K dtype ws ws_bytes stream
FWD = [P, P, P, P, P, P, P, P, 4, 4, 8, 2, 3, 0, P, BIG, None]
# x w tags logp state dlogp dentropy dx dw | N D V T dtype ws ws_bytes stream
BWD = [P] * 9 + [4, 4, 8, 2, 1, P, BIG, None]


def test_logp_refusals():
    f, b = caller(L().logp_fwd, FWD), caller(L().logp_bwd, BWD)
    for i, v in ((8, -1), (8, 1 << 25), (9, 0), (10, 0), (10, 1 << 21), (11, -1), (11, 65), (12, -1), (12, 65), (12, 9), (13, 2)):
        assert f(i, v) == B.LC_EINVAL, (i, v)
    for i in (0, 1, 2, 3, 5, 6):
        assert f(i, None) == B.LC_ENULL, i
    for i in (0, 1, 3, 4, 5, 6, 7, 14):
        assert f(i, P + 8) == B.LC_EALIGN, i
    assert f(2, P + 4) == B.LC_EALIGN
    assert f(14, None) == B.LC_EWORKSPACE and f(15, 8) == B.LC_EWORKSPACE
    a = list(FWD)
    a[2], a[15] = P + 8, 8       # alignment comes before scratch among the checks: any row of a list of tags gets past it
    assert L().logp_fwd(*a) == B.LC_EWORKSPACE
    a = list(FWD)
    a[0] = a[2] = a[3] = a[4] = a[5] = a[6] = a[7] = None
    a[8] = 0
    assert L().logp_fwd(*a) == B.LC_OK      # no rows: nothing to do
    for i, v in ((9, -1), (10, 0), (11, 0), (12, 65), (13, 7)):
        assert b(i, v) == B.LC_EINVAL, (i, v)
    for i in (0, 1, 2, 3, 4, 5, 8):
        assert b(i, None) == B.LC_ENULL, i
    for i in (0, 1, 3, 4, 5, 6, 7, 8, 14):
        assert b(i, P + 8) == B.LC_EALIGN, i
    assert b(2, P + 2) == B.LC_EALIGN
    assert b(14, None) == B.LC_EWORKSPACE and b(15, lc.logp_workspace_bytes(4, 4, 8, 2, 0, 1, True) - 1) == B.LC_EWORKSPACE


def test_muon_refusals():
    # w g m w_out m_out | count rows cols rate decay momentum nesterov steps dtype ws ws_bytes stream
    f = caller(L().muon_step, [P] * 5 + [2, 8, 8, 0.1, 0.0, 0.9, 1, 5, 0, P, BIG, None])
    for i, v in ((5, -1), (5, 1 << 25), (6, 0), (7, 0), (6, 1 << 21), (12, 0), (12, 33), (13, 2), (8, float("nan")), (9, float("inf")), (10, float("nan"))):
        assert f(i, v) == B.LC_EINVAL, (i, v)
    for i in range(5):
        assert f(i, None) == B.LC_ENULL and f(i, P + 4) == B.LC_EALIGN
    assert f(14, P + 8) == B.LC_EALIGN and f(14, None) == B.LC_EWORKSPACE
    assert f(15, lc.muon_workspace_bytes(2, 8, 8) - 1) == B.LC_EWORKSPACE
    assert lc.muon_workspace_bytes(1, (1 << 15) + 1, (1 << 15) + 1) == 0      # the smaller side is bounded
    assert lc.muon_workspace_bytes(1, 1 << 20, 1 << 15) > 0
    assert lc.muon_workspace_bytes(1 << 24, 1 << 10, 1 << 10) == 0            # 2^44 values
    e = [None] * 5 + [0, 8, 8, 0.1, 0.0, 0.9, 1, 5, 0, P, BIG, None]
    assert L().muon_step(*e) == B.LC_OK


def test_q8_refusals():
    assert [lc.q8_row_bytes(d) for d in (1, 128, 129, 1 << 17)] == [128, 128, 256, 1 << 17]
    assert lc.q8_row_bytes(0) == 0 and lc.q8_row_bytes((1 << 17) + 1) == 0
    f = caller(L().q8_rows, [P, P, P, 3, 5, 0, None])
    for i, v in ((3, -1), (4, 0), (4, (1 << 17) + 1), (5, 2)):
        assert f(i, v) == B.LC_EINVAL
    for i in range(3):
        assert f(i, None) == B.LC_ENULL and f(i, P + 8) == B.LC_EALIGN
    assert f(3, 0) == B.LC_OK
    # x q scale y | N D F dtype ws ws_bytes stream
    f = caller(L().q8_matmul, [P] * 4 + [3, 5, 7, 1, P, BIG, None])
    for i, v in ((4, -1), (5, 0), (5, (1 << 17) + 1), (6, 0), (6, 1 << 21), (7, 2)):
        assert f(i, v) == B.LC_EINVAL
    for i in range(4):
        assert f(i, None) == B.LC_ENULL and f(i, P + 8) == B.LC_EALIGN
    assert f(8, None) == B.LC_EWORKSPACE and f(9, lc.q8_workspace_bytes(3, 5, 7, 1) - 1) == B.LC_EWORKSPACE and f(8, P + 2) == B.LC_EALIGN
    assert f(4, 0) == B.LC_OK
    # x qg sg qu su h | N D F act dtype ws ws_bytes stream
    f = caller(L().q8_glu_fwd, [P] * 6 + [3, 5, 7, 1, 1, P, BIG, None])
    for i, v in ((6, -1), (7, 0), (8, 0), (9, 3), (10, 2)):
        assert f(i, v) == B.LC_EINVAL
    for i in range(6):
        assert f(i, None) == B.LC_ENULL and f(i, P + 8) == B.LC_EALIGN
    assert f(11, None) == B.LC_EWORKSPACE and f(12, 100) == B.LC_EWORKSPACE
    assert f(6, 0) == B.LC_OK


def test_the_binding_refuses():
    x, w = torch.zeros(2, 4), torch.zeros(3, 4)
    for call in (lambda: lc.logp_fwd(x, w, None, None, None, None, None, None), lambda: lc.muon_step(w, w, w, None, None, 0.1),
                 lambda: lc.q8_rows(x, torch.zeros(2, 128, dtype=torch.int8), torch.zeros(2)),
                 lambda: lc.q8_matmul(x, torch.zeros(3, 128, dtype=torch.int8), torch.zeros(3), torch.zeros(2, 3))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_any_size_passes_the_host_checks(dtype):
    """Plans of sizes drawn over the whole range, with exactly the scratch that is asked for.  Every check of a launch is applied."""
    rng = random.Random(7)
    for _ in range(1200):
        N, D, V = log_int(rng, 1, 30000), log_int(rng, 1, 16384), log_int(rng, 1, 300000)
        for op in (B.LC_HEAD_LOGP_FWD, B.LC_HEAD_LOGP_BWD, B.LC_HEAD_Q8_MATMUL, B.LC_HEAD_Q8_GLU_FWD):
            lc.head_plan_query(op, N, D, V, dtype)
        rows, cols = log_int(rng, 1, 30000), log_int(rng, 1, 30000)
        lc.head_plan_query(B.LC_HEAD_MUON, log_int(rng, 1, min(1 << 24, max(1, (1 << 30) // (rows * cols)))), rows, cols, dtype)
    for N, D, V in ((1, 1, 1), (1 << 24, 1, 1), (33, 1 << 17, 1 << 20), (1, 1 << 17, 1 << 20)):
        for op in (B.LC_HEAD_LOGP_FWD, B.LC_HEAD_LOGP_BWD, B.LC_HEAD_Q8_MATMUL):
            if N * V <= 1 << 36:
                lc.head_plan_query(op, N, D, V, dtype)
    for c, r, k in ((1, 1 << 20, 1), (1, 1, 1 << 20), (1 << 20, 1, 1), (1, 1 << 15, 1 << 15), (3, 1 << 20, 1 << 10), (100000, 16, 16)):
        lc.head_plan_query(B.LC_HEAD_MUON, c, r, k, dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_parts_fit_what_is_set_aside(dtype):
    """Counted apart from the sources: a cut product's parts, [items][parts][rows][columns to a multiple of 4] floats, and the planes."""
    rng = random.Random(8)
    planes = 2 if dtype == lc.LC_F32 else 1
    seen = 0
    for _ in range(600):
        rows, cols = log_int(rng, 1, 20000), log_int(rng, 1, 20000)
        count = log_int(rng, 1, min(1 << 24, max(1, (1 << 27) // (rows * cols))))
        plans = lc.head_plan_query(B.LC_HEAD_MUON, count, rows, cols, dtype)
        cut = [p["arg"] for p in plans if p["kernel"].startswith("muon_step (") and p["tparam"][3] in (64, 128, 192, 256) and p["arg"][3] > 1]
        parts = max([4 * a[0] * up(a[1], 4) * a[3] * a[4] for a in cut], default=0)
        seen += parts > 0
        items = max(p["arg"][4] for p in plans if p["kernel"].startswith("muon_step (") and p["tparam"][3] in (32, 64, 128, 192, 256))
        small = min(rows, cols)
        used = parts + items * planes * 2 * (2 * rows * up(cols, 8) + 2 * small * up(small, 8))
        assert used <= lc.muon_workspace_bytes(count, rows, cols, dtype), (count, rows, cols)
    assert seen > 20


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_scratch_for_many_is_enough_for_fewer(dtype):
    rng = random.Random(9)
    for _ in range(150):
        N, D, V = log_int(rng, 2, 8192), log_int(rng, 1, 8192), log_int(rng, 1, 200000)
        for T in (0, 2):
            fwd, both = (lc.logp_workspace_bytes(N, D, V, T, 1, dtype, g) for g in (False, True))
            assert fwd <= both
            assert all(lc.logp_workspace_bytes(N, D, V, T, k, dtype) <= lc.logp_workspace_bytes(N, D, V, T, min(V, 40), dtype) for k in range(min(V, 40)))
            for n in {rng.randrange(N) for _ in range(40)} | set(range(min(N, 40))):
                assert lc.logp_workspace_bytes(n, D, V, T, 1, dtype) <= fwd and lc.logp_workspace_bytes(n, D, V, T, 1, dtype, True) <= both, (n, N, D, V)
        assert all(lc.q8_workspace_bytes(n, D, V, dtype) <= lc.q8_workspace_bytes(N, D, V, dtype) for n in range(0, N, 37))
        rows, cols = log_int(rng, 1, 8192), log_int(rng, 1, 8192)
        count = log_int(rng, 2, 3000)
        most = lc.muon_workspace_bytes(count, rows, cols, dtype)
        assert all(lc.muon_workspace_bytes(n, rows, cols, dtype) <= most for n in {rng.randrange(count) for _ in range(40)} | {0, 1, count - 1}), (count, rows, cols)


def test_scratch_is_bounded():
    """Neither rows by words without bound, nor a stack's planes."""
    a, b = (lc.logp_workspace_bytes(n, 64, 100000, 0, 5, lc.LC_BF16, True) for n in (1 << 17, 1 << 18))
    assert b - a < 1 << 30 and a < 5 << 30
    assert lc.muon_workspace_bytes(1 << 20, 128, 128) < 12 << 30


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_square_matrices_take_one_step_at_a_time(dtype):
    """Neither side is the shorter one: the products and places of several steps on the short side alone (P A, P A P, Q) are for others."""
    for count, n in [(c, n) for c in (1, 2, 3, 5, 7, 9, 24, 100) for n in (129, 256, 513, 1281, 1477, 2048, 2499, 2816, 2950, 3270, 4096, 4291, 5120, 7680, 8192)]:
        if count * n * n > 1 << 31:
            continue
        names = [p["kernel"] for p in lc.head_plan_query(B.LC_HEAD_MUON, count, n, n, dtype)]
        assert "muon_step (X)" in names and not {"muon_step (P A)", "muon_step (P A P)", "muon_step (Q)"} & set(names), (count, n)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_most_rows_and_matrices_can_be_launched(dtype):
    """A launch takes fewer than 2^32 threads."""
    for N in (1 << 23, (1 << 23) + 1, (1 << 24) - 1, 1 << 24):
        plans = [lc.head_plan_query(op, N, 1, 2, dtype) for op in (B.LC_HEAD_LOGP_FWD, B.LC_HEAD_LOGP_BWD, B.LC_HEAD_Q8_MATMUL, B.LC_HEAD_Q8_GLU_FWD)]
        plans += [lc.head_plan_query(B.LC_HEAD_MUON, N, r, c, dtype) for r, c in ((1, 1), (3, 8), (9, 5))]
        for p in sum(plans, []):
            assert p["grid"][0] * p["grid"][1] * p["grid"][2] * p["block"] < 1 << 32, (N, p)
