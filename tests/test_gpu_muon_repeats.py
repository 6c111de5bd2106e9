"""muon_step where symmetric products take tiles of 256 x 256, which eight waves share: against its definition, and the same bits from call to
call, with results in their own places and in place."""
import pytest
import torch

import paper_1502_03409_amd as lc
import test_gpu_muon as MU
from paper_1502_03409_amd import binding as B
from test_head_tiles_host import LARGE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", MU.TYPES, ids=MU.ids)
@pytest.mark.parametrize("shape", LARGE, ids=str)
def test_calls_repeat_bit_by_bit(shape, dtype):
    print(f"case muon repeated {shape} {dtype}", flush=True)
    w, g, m = (torch.empty(shape, device="cuda").normal_(0, std, generator=torch.Generator("cuda").manual_seed(k)) for k, std in enumerate((2.0 ** -6, 1.0, 4.0)))
    w, g = w.to(dtype), g.to(dtype)
    first = MU.step(w, g, m)
    for in_place in (False, True, False, False):
        again = MU.step(w, g, m, in_place=in_place)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    MU.check(first, w, g, m, bounds=True)


def test_a_stack_that_is_taken_in_parts():
    """Nearly square matrices, whose squares fill the scratch: the first and last of each part, the last part shorter."""
    shape = n, rows, cols = 700, 600, 601
    print(f"case muon in parts {shape}", flush=True)
    plans = [p for p in lc.head_plan_query(B.LC_HEAD_MUON, *shape) if p["kernel"] == "muon_momentum"]
    counts = [p["arg"][0] for p in plans]
    assert len(counts) > 1 and sum(counts) == n and counts[-1] < counts[0]
    w, g, m = (torch.empty(shape, device="cuda").normal_(0, std, generator=torch.Generator("cuda").manual_seed(k)) for k, std in enumerate((2.0 ** -6, 1.0, 4.0)))
    at = sorted({0, n - 1} | {sum(counts[:k]) + d for k in range(1, len(counts)) for d in (-1, 0)})
    got = MU.step(w, g, m)
    MU.check((got[0][at], got[1][at]), w[at], g[at], m[at], bounds=True)
