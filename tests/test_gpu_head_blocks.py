"""Cross entropy over more rows than are kept at a time, where the last block's products are cut otherwise than the full blocks'."""
import pytest
import torch

import head_ref as ref
import paper_1502_03409_amd as lc
import test_gpu_xent as X
from paper_1502_03409_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,N,D,V", [(torch.bfloat16, 6625, 66, 247098), (torch.float32, 10657, 66, 80377)], ids=["bf16", "f32"])
def test_a_short_last_block_of_more_parts(dtype, N, D, V):
    """The last block's parts are more floats than those of a full block, and dw adds up over both."""
    print(f"case xent short last block {N} {D} {V} {dtype}", flush=True)
    plans = lc.head_plan_query(B.LC_HEAD_XENT_FWD_BWD, N, D, V, X.code(dtype))
    parts = [[p["arg"][0] * (p["arg"][3] > 1) * p["arg"][3] for p in plans if p["kernel"] == name and p["tparam"][3]]
             for name in ("xent (dx)", "xent (dw)")]
    assert len(parts[0]) == 2 and max(p[1] for p in parts) > max(p[0] for p in parts)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((N, D), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((V, D), generator=gen, device="cuda") * 2 * D ** -0.5).to(dtype)
    t = torch.randint(0, V, (N,), generator=gen, device="cuda")
    t[torch.rand(N, generator=gen, device="cuda") < 0.1] = -1
    loss, cost, dx, dw = X.run(x, w, t)
    rx, rw, rl = torch.empty(N, D, device="cuda", dtype=torch.float64), torch.zeros(V, D, device="cuda", dtype=torch.float64), []
    count = int((t >= 0).sum())
    for i in range(0, N, 1000):
        s = torch.full((min(1000, N - i),), 1.0 / count, device="cuda")
        l, _, a, b = ref.xent(x[i:i + 1000], w, t[i:i + 1000], s)
        rl.append(l)
        rx[i:i + 1000] = a
        rw += b
    b = X.loss_bound(x.float(), w)
    assert float((loss.double() - torch.cat(rl)).abs().max()) <= b
    bound = ref.tol(dtype, V, 2.25) + b
    ref.check("dx", dx, rx, bound)
    ref.check("dw", dw, rw, bound)
