"""muon_step where symmetric products take tiles of 256 x 256, which eight waves share: against its definition, and the same bits from call to
call, with results in their own places and in place."""
import pytest
import torch

import test_gpu_muon as MU
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
