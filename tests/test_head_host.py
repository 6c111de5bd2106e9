"""The supervised head's entry points on the host: every symbol of the header is there, and arguments are refused before
anything is launched."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_1502_03409_amd as lc
from paper_1502_03409_amd import binding as B
from paper_1502_03409_amd import head as H

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000      # an aligned address that is never used: every call below is refused, or has nothing to do
BIG = 1 << 50    # a workspace size that is always enough


def L():
    return H._lib()


def test_every_declared_symbol_is_exported():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lc_head.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(?:int|size_t)\s+(\w+)\s*\(", src))
    assert names == set(H.HEAD_EXPORTS)
    for n in names:
        assert hasattr(L(), n) and hasattr(lc, n), n


def test_workspace_sizes():
    assert lc.glu_workspace_bytes(0, 5, 7) > 0
    for bad in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), (1 << 25, 4, 4), (4, 1 << 21, 4), (4, 4, 1 << 21)):
        assert lc.glu_workspace_bytes(*bad) == 0
        assert lc.xent_workspace_bytes(*bad) == 0
    assert lc.glu_workspace_bytes(4, 4, 4, 7) == 0 and lc.xent_workspace_bytes(4, 4, 4, 7) == 0
    for dtype in (lc.LC_F32, lc.LC_BF16):
        assert lc.glu_workspace_bytes(64, 64, 64, dtype, True) >= lc.glu_workspace_bytes(64, 64, 64, dtype)
        assert lc.xent_workspace_bytes(64, 64, 64, dtype, True) >= lc.xent_workspace_bytes(64, 64, 64, dtype)
    # the loss alone keeps no array of rows by words; with gradients the exponentials are kept for a bounded number of rows
    assert lc.xent_workspace_bytes(8192, 64, 100000, lc.LC_BF16) < 8192 * 100000 // 4
    a, b = (lc.xent_workspace_bytes(n, 64, 100000, lc.LC_BF16, True) for n in (1 << 17, 1 << 18))
    assert b - a < 1 << 30
    assert L().grad_clip_workspace_bytes(-1, 3) == 0 and L().grad_clip_workspace_bytes(3, -1) == 0
    assert L().grad_clip_workspace_bytes(0, 0) > 0


def test_glu_refusals():
    f, b = L().glu_fwd, L().glu_bwd
    ok = [P, P, P, P, None, 4, 4, 4, 0, 0, P, BIG, None]

    def fwd(i, v):
        a = list(ok)
        a[i] = v
        return f(*a)

    for i, v in ((5, -1), (6, 0), (7, 0), (7, 1 << 21), (8, 3), (8, -1), (9, 2)):
        assert fwd(i, v) == B.LC_EINVAL
    for i in (0, 1, 2, 3):
        assert fwd(i, None) == B.LC_ENULL
        assert fwd(i, P + 8) == B.LC_EALIGN
    assert fwd(4, P + 4) == B.LC_EALIGN and fwd(10, P + 2) == B.LC_EALIGN
    assert fwd(10, None) == B.LC_EWORKSPACE and fwd(11, 1) == B.LC_EWORKSPACE
    assert f(None, P, P, None, None, 0, 4, 4, 0, 0, P, BIG, None) == B.LC_OK      # no rows: nothing to do
    okb = [P] * 8 + [4, 4, 4, 1, 1, P, BIG, None]

    def bwd(i, v):
        a = list(okb)
        a[i] = v
        return b(*a)

    for i in (0, 1, 2, 3, 4, 6, 7):
        assert bwd(i, None) == B.LC_ENULL
    for i in range(8):
        assert bwd(i, P + 2) == B.LC_EALIGN
    assert bwd(11, 9) == B.LC_EINVAL and bwd(12, 9) == B.LC_EINVAL
    assert bwd(14, lc.glu_workspace_bytes(4, 4, 4, 1, True) - 1) == B.LC_EWORKSPACE


def test_xent_refusals():
    f, b = L().xent_fwd, L().xent_fwd_bwd
    ok = [P, P, P, None, P, P, 4, 4, 4, 0, P, BIG, None]

    def fwd(i, v):
        a = list(ok)
        a[i] = v
        return f(*a)

    for i, v in ((6, -1), (7, 0), (8, 0), (9, 5)):
        assert fwd(i, v) == B.LC_EINVAL
    for i in (0, 1, 2, 4, 5):
        assert fwd(i, None) == B.LC_ENULL
    for i in (0, 1, 2, 3, 4, 5, 10):
        assert fwd(i, P + 4) == B.LC_EALIGN
    assert fwd(10, None) == B.LC_EWORKSPACE and fwd(11, 8) == B.LC_EWORKSPACE
    okb = [P, P, P, P, P, P, P, P, 4, 4, 4, 1, P, BIG, None]

    def bwd(i, v):
        a = list(okb)
        a[i] = v
        return b(*a)

    assert bwd(7, None) == B.LC_ENULL and bwd(6, P + 8) == B.LC_EALIGN
    assert bwd(13, lc.xent_workspace_bytes(4, 4, 4, 1, True) - 1) == B.LC_EWORKSPACE


def test_grad_clip_refusals():
    f = L().grad_clip

    def call(src=P, dst=P, n=10, dtype=0, max_norm=1.0, norm=P, ws=P, wsb=BIG, count=1):
        words = (C.c_uint64 * 4)(src, dst, n & (2 ** 64 - 1), dtype)
        return f(words, count, max_norm, norm, ws, wsb, None)

    assert call(n=-1) == B.LC_EINVAL and call(dtype=2) == B.LC_EINVAL and call(n=1 << 41) == B.LC_EINVAL
    for bad in (0.0, -1.0, float("nan")):
        assert call(max_norm=bad) == B.LC_EINVAL
    assert call(src=0) == B.LC_ENULL and call(dst=0) == B.LC_ENULL and call(norm=None) == B.LC_ENULL
    assert call(src=P + 2) == B.LC_EALIGN and call(src=P + 1, dtype=1) == B.LC_EALIGN and call(dst=P + 2) == B.LC_EALIGN
    assert call(norm=P + 2) == B.LC_EALIGN and call(ws=P + 8) == B.LC_EALIGN
    assert call(ws=None) == B.LC_EWORKSPACE and call(wsb=7) == B.LC_EWORKSPACE
    assert call(count=-1) == B.LC_EINVAL
    assert f(None, 1, 1.0, P, P, BIG, None) == B.LC_ENULL


def test_the_binding_refuses():
    x, w = torch.zeros(2, 4), torch.zeros(3, 4)
    with pytest.raises(ValueError):
        lc.glu_fwd(x, w, w, torch.zeros(2, 3), None, lc.LC_ACT_SILU)
    with pytest.raises(ValueError):
        lc.grad_clip([x], [x, w], 1.0, torch.zeros(1))
    with pytest.raises(ValueError):
        lc.grad_norm([torch.zeros(3, dtype=torch.float64)], torch.zeros(1))
    with pytest.raises(ValueError):
        lc.grad_norm([x], torch.zeros(1))


def test_targets_may_start_at_any_row_of_a_list():
    """Alignment comes before scratch among the checks: a target aligned to 8 bytes gets past it, an odd one does not."""
    for target, code in ((P + 8, B.LC_EWORKSPACE), (P + 24, B.LC_EWORKSPACE), (P + 4, B.LC_EALIGN), (P + 1, B.LC_EALIGN)):
        assert L().xent_fwd(P, P, target, None, P, P, 4, 4, 4, 0, P, 8, None) == code
        assert L().xent_fwd_bwd(P, P, target, P, P, P, P, P, 4, 4, 4, 1, P, 8, None) == code
